"""Rotary positions of several axes against the formula in float64, and against the call of one axis."""
import math

import numpy as np
import pytest
import torch

from tests.kv_ranges_testlib import TYPES, half_step, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def by_turns(pairs, n):
    return (np.arange(pairs) % n).astype(np.int32)


def by_sections(pairs, n):
    return (np.arange(pairs) * n // pairs).astype(np.int32)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows, nq, nk, hd, rot, n, order", [
    (1, 2, 1, 128, 128, 3, by_sections), (37, 32, 8, 128, 128, 3, by_turns), (5, 3, 3, 64, 32, 2, by_sections), (9, 2, 1, 80, 20, 4, by_turns),
    (3, 1, 0, 256, 256, 8, by_turns), (4, 0, 2, 7, 6, 3, by_turns), (130, 4, 4, 64, 64, 1, by_turns)])
def test_rope_axes(R, layout, dt, rows, nq, nk, hd, rot, n, order):
    dtype, h = TYPES[dt], rot // 2
    wide = randn(rows + hd, rows, (nq + nk + 1) * hd + 8 - (nq + nk + 1) * hd % 8, dtype=dtype)
    q = wide[:, :nq * hd].view(rows, nq, hd) if nq else None
    k = wide[:, nq * hd:(nq + nk) * hd].view(rows, nk, hd) if nk else None
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (n, rows), generator=torch.Generator().manual_seed(rows), dtype=torch.int64).int()
    pos[:, 0] = torch.arange(n)
    freqs, _ = R.riftkv_rope_freqs(rot)
    axes = order(h, n)
    outs = [None if x is None else torch.full((rows, m, hd), 5.0, dtype=dtype, device="cuda") for x, m in ((q, nq), (k, nk))]
    before = wide.clone()
    R.riftkv_rope_axes(q, k, pos.cuda(), freqs, axes, *outs, layout=layout, magnitude=1.25)
    assert torch.equal(wide, before)
    a = pos.double()[torch.from_numpy(axes).long()].t() * torch.from_numpy(freqs)   # [rows][pairs]
    # far positions: the product's 53 bits are not enough for a reference, the angle is reduced exactly there
    exact = np.empty(a.shape)
    for i in range(rows):
        for j in range(h):
            p, f = int(pos[axes[j], i]), float(freqs[j])
            num, den = f.as_integer_ratio()
            exact[i, j] = reduced(p * num, den)
    c, s = (torch.from_numpy(fn(exact) * 1.25)[:, None] for fn in (np.cos, np.sin))
    for x, o in zip((q, k), outs):
        if x is None:
            continue
        y = x.double().cpu()
        i1 = torch.arange(h) if layout == "half" else 2 * torch.arange(h)
        i2 = i1 + h if layout == "half" else i1 + 1
        x1, x2 = y[..., i1].clone(), y[..., i2].clone()
        # the angle's rounding (pi 2^-25), sine and cosine (2 steps), magnitude, product and sum (4 half steps)
        e = (x1.abs() + x2.abs()) * 1.25 * (math.pi * 2.0 ** -25 + 2 * 2.0 ** -23 + 4 * 2.0 ** -24)
        y[..., i1], y[..., i2] = x1 * c - x2 * s, x2 * c + x1 * s
        err = torch.zeros_like(y)
        err[..., i1] = err[..., i2] = e
        off = (o.double().cpu() - y).abs()
        assert bool((off <= err + half_step(dtype) * y.abs() * (1 + 1e-3) + 1e-30).all())
        assert torch.equal(o[..., rot:], x[..., rot:])
    R.riftkv_rope_axes(q, k, pos.cuda(), freqs, axes, layout=layout, magnitude=1.25)   # in place: the same bits
    for x, o in zip((q, k), outs):
        assert x is None or torch.equal(x, o)
    assert torch.equal(wide[:, (nq + nk) * hd:], before[:, (nq + nk) * hd:])


def reduced(num, den):
    """num / den reduced by whole turns of 2 pi, in integers of 300 bits."""
    bits = 300
    two_pi = TWO_PI >> (TWO_PI_BITS - bits)
    x = (num << bits) // den
    x -= two_pi * round_div(x, two_pi)
    return x / (1 << bits)


def round_div(a, b):
    return (2 * a + b) // (2 * b)


def arctan_inverse(n, bits):
    """arctan(1 / n) 2^bits by its series."""
    x = (1 << bits) // n
    total, k, sign = x, 1, 1
    while x:
        x //= n * n
        k += 2
        sign = -sign
        total += sign * (x // k)
    return total


TWO_PI_BITS = 400
TWO_PI = 2 * 4 * (4 * arctan_inverse(5, TWO_PI_BITS + 20) - arctan_inverse(239, TWO_PI_BITS + 20)) >> 20


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd, rot", [(128, 128), (64, 32), (20, 12)])
def test_one_position_on_all_axes(R, layout, hd, rot):
    """riftkv_rope's bits."""
    rows = 50
    q, k = randn(1, rows, 4, hd), randn(2, rows, 2, hd)
    pos = torch.randint(0, 1 << 20, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    freqs, _ = R.riftkv_rope_freqs(rot)
    one = torch.empty_like(q), torch.empty_like(k)
    R.riftkv_rope(q, k, pos, freqs, *one, layout=layout)
    for n in (1, 3):
        all_axes = torch.empty_like(q), torch.empty_like(k)
        R.riftkv_rope_axes(q, k, pos.expand(n, rows).contiguous(), freqs, by_turns(rot // 2, n), *all_axes, layout=layout)
        assert torch.equal(one[0], all_axes[0]) and torch.equal(one[1], all_axes[1])


def test_axes_in_a_graph_and_on_a_stream(R):
    rows = 33
    q, k = randn(1, rows, 4, 128), randn(2, rows, 2, 128)
    pos = torch.randint(0, 4096, (3, rows), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    freqs, _ = R.riftkv_rope_freqs(128)
    axes = by_turns(64, 3)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    R.riftkv_rope_axes(q, k, pos, freqs, axes, qo, ko)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.riftkv_rope_axes(q, k, pos, freqs, axes, qo, ko)
    axes[:] = 0                                              # read before the call returned
    freqs[:] = 0
    axes2, freqs2 = by_turns(64, 3), R.riftkv_rope_freqs(128)[0]
    side = torch.cuda.Stream()
    for i in range(3):
        pos.copy_(torch.randint(0, 4096, (3, rows), generator=torch.Generator().manual_seed(5 + i), dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b = qo.clone(), ko.clone()
        qo.zero_(), ko.zero_()
        torch.cuda.synchronize()
        R.riftkv_rope_axes(q, k, pos, freqs2, axes2, qo, ko, stream=side)
        side.synchronize()
        assert torch.equal(a, qo) and torch.equal(b, ko)


def test_rows_of_no_length(R):
    freqs, _ = R.riftkv_rope_freqs(64)
    x = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    R.riftkv_rope_axes(x, None, torch.empty(2, 0, dtype=torch.int32, device="cuda"), freqs, by_turns(32, 2))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows, nq, nk, hd, rot", [
    (1025, 1, 0, 16, 16), (16389, 1, 0, 16, 16), (4099, 0, 1, 64, 32), (2051, 2, 1, 64, 64), (20001, 1, 1, 64, 64), (1030, 3, 1, 128, 128),
    (2100, 8, 2, 128, 128), (2049, 1, 1, 256, 256), (4100, 1, 2, 128, 16), (1100, 16, 16, 64, 64)])
def test_many_rows_of_few_heads(R, layout, dt, rows, nq, nk, hd, rot):
    """Many rows of few heads share workgroups, few do not: the same bits either way, on one axis and on several, in place
    and not, with the row behind the last left as it was."""
    dtype = TYPES[dt]
    wide = randn(rows + nq, rows + 1, (nq + nk) * hd, dtype=dtype)
    g = torch.Generator().manual_seed(hd)
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (3, rows), generator=g, dtype=torch.int64).int().cuda()
    freqs, _ = R.riftkv_rope_freqs(rot)
    axes = by_turns(rot // 2, 3)

    def parts(t, n):
        return (t[:n, :nq * hd].view(n, nq, hd) if nq else None, t[:n, nq * hd:].view(n, nk, hd) if nk else None)

    for several in (True, False):
        def call(t, n, places):
            q, k = parts(t, n)
            if several:
                R.riftkv_rope_axes(q, k, places.contiguous(), freqs, axes, layout=layout)
            else:
                R.riftkv_rope(q, k, places[0].contiguous(), freqs, layout=layout)

        want, got, out = wide.clone(), wide.clone(), wide.clone()
        for r in range(0, rows, 300):
            n = min(300, rows - r)
            call(want[r:r + n], n, pos[:, r:r + n])
        call(got, rows, pos)
        assert torch.equal(got, want) and torch.equal(got[rows], wide[rows]) and not torch.equal(got, wide)
        out.fill_(7.0)
        args = (*parts(wide, rows), pos if several else pos[0], freqs)
        outs = parts(out, rows)
        if several:
            R.riftkv_rope_axes(*args, axes, *outs, layout=layout)
        else:
            R.riftkv_rope(*args, *outs, layout=layout)
        assert torch.equal(out[:rows], want[:rows]) and bool((out[rows] == 7.0).all())
