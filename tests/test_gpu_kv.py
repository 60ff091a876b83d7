"""The paged key-value cache's kernels against plain float64 forms."""
import math

import numpy as np
import pytest
import torch

from tests.kv_testlib import LARGEST, STORES, Pages, attend, half_step, quantise

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def randn(seed, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


# ----------------------------------------------------------------------------- positions
def rope_ref(x, pos, freqs, rot, layout, mag):
    """float64 rotation and the float32 evaluation's error: |x1| + |x2| times the angle's
    rounding (pi 2^-25), sine and cosine (2 steps), magnitude, product and sum (3 half steps)."""
    y = x.double().cpu().clone()
    a = pos.double().cpu()[:, None] * torch.from_numpy(freqs)[None]
    c, s = (torch.cos(a) * mag)[:, None], (torch.sin(a) * mag)[:, None]
    h = rot // 2
    i1 = torch.arange(h) if layout == "half" else 2 * torch.arange(h)
    i2 = i1 + h if layout == "half" else i1 + 1
    x1, x2 = y[..., i1].clone(), y[..., i2].clone()
    err = torch.zeros_like(y)
    e = (x1.abs() + x2.abs()) * abs(mag) * (math.pi * 2.0 ** -25 + 2 * 2.0 ** -23 + 4 * 2.0 ** -24)
    y[..., i1], y[..., i2] = x1 * c - x2 * s, x2 * c + x1 * s
    err[..., i1] = err[..., i2] = e
    return y, err


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows, nq, nk, hd, rot", [(1, 1, 1, 64, 64), (7, 32, 8, 128, 128), (130, 4, 1, 128, 64),
                                                   (33, 3, 3, 128, 32), (5, 2, 1, 80, 20), (9, 2, 2, 256, 256),
                                                   (4, 3, 1, 7, 6), (17, 5, 0, 64, 2), (64, 0, 2, 64, 16), (3, 6, 2, 96, 96)])
def test_rope(R, layout, dt, rows, nq, nk, hd, rot):
    """Slices of a projection with a tail of values, positions far, near and negative,
    into new rows and in place; nothing beside the rows changes."""
    dtype = TYPES[dt]
    wide = randn(rows + hd, rows, (nq + nk + 1) * hd + 8 - (nq + nk + 1) * hd % 8, dtype=dtype)
    q = wide[:, :nq * hd].view(rows, nq, hd) if nq else None
    k = wide[:, nq * hd:(nq + nk) * hd].view(rows, nk, hd) if nk else None
    g = torch.Generator().manual_seed(rows)
    pos = torch.randint(0, 1 << 20, (rows,), generator=g, dtype=torch.int32)
    pos[0] = 0
    pos[-1] = 2 ** 31 - 1 if rows > 1 else 5
    if rows > 4:
        pos[1:3] = torch.tensor([-1, -70000])
    freqs, _ = R.riftkv_rope_freqs(rot)
    mag = 1.25
    qo = None if q is None else torch.empty(rows, nq, hd, dtype=dtype, device="cuda")
    ko = None if k is None else torch.empty(rows, nk, hd, dtype=dtype, device="cuda")
    before = wide.clone()
    R.riftkv_rope(q, k, pos.cuda(), freqs, qo, ko, layout=layout, magnitude=mag)
    torch.cuda.synchronize()
    assert torch.equal(wide, before)
    for x, o in ((q, qo), (k, ko)):
        if x is None:
            continue
        ref, err = rope_ref(x, pos, freqs, rot, layout, mag)
        got = o.double().cpu()
        bound = err + half_step(dtype) * ref.abs() * (1 + 1e-3) + 1e-30
        assert bool(((got - ref).abs() <= bound).all()), float(((got - ref).abs() / bound).max())
        assert torch.equal(o[..., rot:], x[..., rot:])
    R.riftkv_rope(q, k, pos.cuda(), freqs, layout=layout, magnitude=mag)   # in place: the same bits
    torch.cuda.synchronize()
    if q is not None:
        assert torch.equal(q, qo)
    if k is not None:
        assert torch.equal(k, ko)
    assert torch.equal(wide[:, (nq + nk) * hd:], before[:, (nq + nk) * hd:])


def test_rope_keeps_nan_and_infinity(R):
    x = randn(3, 2, 1, 64, dtype=torch.bfloat16)
    x[0, 0, 3] = math.nan
    x[1, 0, 5] = math.inf
    o = torch.empty_like(x)
    freqs, _ = R.riftkv_rope_freqs(64)
    R.riftkv_rope(x, None, torch.tensor([1, 1], dtype=torch.int32, device="cuda"), freqs, o)
    o = o.cpu().float()
    assert bool(torch.isnan(o[0, 0, [3, 35]]).all()) and int(torch.isnan(o).sum()) == 2
    assert bool(torch.isinf(o[1, 0, [5, 37]]).all())


# ----------------------------------------------------------------------------- rows
def special_rows(n_kv, hd, dtype):
    """Rows where a scale or a rounding is at a border: [rows][n_kv][hd]."""
    rows = []
    g = torch.Generator().manual_seed(11)
    noise = lambda s=1.0: torch.randn(n_kv, hd, generator=g) * s
    rows.append(torch.zeros(n_kv, hd))
    for top in (448.0, 450.0, 127.0, 127.5, 128.0, 1.0, 2.0 ** -120, 3e38, 2.0 ** 100 * 1.75):
        x = noise().clamp(-1, 1) * top * 0.5
        x[:, 1] = -top
        rows.append(x)
    x = torch.arange(hd).repeat(n_kv, 1).float() / 2 - 15.5                # ties of int8 at scale 1
    x[:, 0] = 127.0
    rows.append(x)
    x = torch.arange(hd).repeat(n_kv, 1).float() * 2.0 ** -10              # subnormal e4m3 codes and their ties
    x[:, 0] = 448.0
    rows.append(x)
    for bad in (math.nan, math.inf, -math.inf):
        x = noise()
        x[n_kv // 2, hd - 1] = bad
        rows.append(x)
    return torch.stack(rows).to(dtype).cuda()


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "bf16"),
                                       ("f32", "fp8"), ("f32", "int8")])
@pytest.mark.parametrize("n_kv, hd, page", [(1, 64, 16), (3, 128, 16), (8, 128, 64), (5, 64, 32)])
def test_write_and_read(R, store, dt, n_kv, hd, page):
    """Several sequences written in one call from strided rows: codes and scale bytes by
    the definition bit for bit, no other byte touched, rows read back in both types."""
    dtype = TYPES[dt]
    lens, first = [1, 2 * page + 3, 16, 5], [0, page - 2, 3, 40]
    P = Pages(R, store, n_kv, hd, page, [n + f for n, f in zip(lens, first)], seed=hd + page)
    sp = special_rows(n_kv, hd, dtype)
    T = sum(lens) + 2
    kv = randn(7, T, 2, n_kv, hd, dtype=dtype)
    m = min(T, sp.shape[0])
    kv[:m, 0] = sp[:m]
    kv[:m, 1] = sp.flip(0)[:m]
    ids, pos = [], []
    for i, (n, f) in enumerate(zip(lens, first)):
        ids += [i] * n
        pos += list(range(f, f + n))
    ids = torch.tensor(ids + [-1, 2], dtype=torch.int32, device="cuda")        # two rows of padding
    pos = torch.tensor(pos + [0, -5], dtype=torch.int32, device="cuda")
    k, v = kv[:, 0], kv[:, 1]
    ref_k, ref_v = (x.view(torch.uint8).clone() for x in (P.k, P.v))
    R.riftkv_write(P.cache, k, v, P.table, pos, P.status, seq_ids=ids)
    torch.cuda.synchronize()
    assert int(P.status) == 0
    page_of = P.table[ids[:-2].long(), pos[:-2].long() // page].long()
    row_of = pos[:-2].long() % page
    size = P.k.element_size()
    for x, pages, scales, ref in ((k, P.k, P.ks, ref_k), (v, P.v, P.vs, ref_v)):
        x = x[:-2]
        if scales is None:
            want = x.to(P.store)
        else:
            code, byte = quantise(x.cpu(), P.store)
            want = code.float().to(P.store).cuda()
            s = torch.full_like(scales, 255)
            s[page_of, :, row_of] = byte.to(torch.uint8).cuda()
            assert torch.equal(scales, s)
        ref.view(*P.k.shape[:3], hd * size)[page_of, :, row_of] = want.contiguous().view(torch.uint8).view(-1, n_kv, hd * size)
        same = pages.view(torch.uint8) == ref.view(pages.view(torch.uint8).shape)
        if scales is None:   # NaN may come back with other bits
            same |= (torch.isnan(pages) & torch.isnan(ref.view(pages.view(torch.uint8).shape).view(P.store))).repeat_interleave(size, -1)
        elif store == "fp8":   # zero has two codes
            same |= ((pages.view(torch.uint8) | ref.view(pages.view(torch.uint8).shape)) & 0x7F) == 0
        assert bool(same.all())
    for out in ("bf16", "f32"):
        o = torch.full((T, 2 * n_kv * hd + 8), 5.0, dtype=TYPES[out], device="cuda")
        ko, vo = (o[:, a:a + n_kv * hd].view(T, n_kv, hd) for a in (0, n_kv * hd))
        R.riftkv_read(P.cache, P.table, pos, ko, vo, P.status, seq_ids=ids)
        torch.cuda.synchronize()
        assert int(P.status) == 0
        assert bool((o[-2:] == 5).all()) and bool((o[:, 2 * n_kv * hd:] == 5).all())   # padding and the gap
        for got, pages, scales in ((ko, P.k, P.ks), (vo, P.v, P.vs)):
            want = pages.view(torch.uint8).view(*P.k.shape[:3], hd * size)[page_of, :, row_of].contiguous().view(P.store).float().double()
            if scales is not None:
                b = scales[page_of, :, row_of].double()
                want = want * torch.where(b == 255, math.nan, torch.pow(2.0, b - 127))[..., None]
            want = want.float().to(TYPES[out]) if out == "bf16" else want.float()
            a, b = got[:-2].float(), want.float()
            assert bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


@pytest.mark.parametrize("store", ["fp8", "int8"])
def test_written_again_gives_the_same_values(R, store):
    """int8: the same bytes too.  e4m3: a largest value just over 448 s is stored at scale 2 s as 224, which
    read back is 448 s: the second write may take the smaller scale, which holds the same values."""
    P = Pages(R, store, 4, 128, 32, [200])
    k, v = randn(1, 200, 4, 128), randn(2, 200, 4, 128, scale=30)
    P.put(R, 0, k, v)
    pos = torch.arange(200, dtype=torch.int32, device="cuda")
    ids = torch.zeros(200, dtype=torch.int32, device="cuda")
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    R.riftkv_read(P.cache, P.table, pos, ko, vo, P.status, seq_ids=ids)
    was = [x.view(torch.uint8).clone() for x in (P.k, P.v, P.ks, P.vs)]
    R.riftkv_write(P.cache, ko, vo, P.table, pos, P.status, seq_ids=ids)
    again = torch.empty_like(k), torch.empty_like(v)
    R.riftkv_read(P.cache, P.table, pos, *again, P.status, seq_ids=ids)
    torch.cuda.synchronize()
    assert torch.equal(again[0], ko) and torch.equal(again[1], vo)
    if store == "int8":
        for a, b in zip(was, (P.k, P.v, P.ks, P.vs)):
            assert torch.equal(a, b.view(torch.uint8))


@pytest.mark.parametrize("store", ["bf16", "fp8"])
def test_rows_out_of_range(R, store):
    """Bad sequences, positions and pages: the status set, their rows skipped, the others there."""
    P = Pages(R, store, 2, 64, 16, [20, 20])
    bad_table = P.table.clone()
    bad_table[1, 1] = P.k.shape[0]            # one past the pool
    k, v = randn(1, 7, 2, 64), randn(2, 7, 2, 64)
    ids = torch.tensor([0, 2, 0, 1, 1, 0, 1], dtype=torch.int32, device="cuda")
    pos = torch.tensor([3, 0, 32, 16, 5, 2 ** 31 - 1, 17], dtype=torch.int32, device="cuda")
    R.riftkv_write(P.cache, k, v, bad_table, pos, P.status, seq_ids=ids)
    torch.cuda.synchronize()
    assert int(P.status) == 2
    written = ~(P.k.view(torch.uint8) == 255).all(-1).all(1)      # [n_pages][page]
    assert int(written.sum()) == 2
    assert bool(written[P.table[0, 0].long(), 3]) and bool(written[P.table[1, 0].long(), 5])
    P.status.zero_()
    ko, vo = torch.full_like(k, 5), torch.full_like(v, 5)
    R.riftkv_read(P.cache, bad_table, pos, ko, vo, P.status, seq_ids=ids)
    torch.cuda.synchronize()
    assert int(P.status) == 2
    kept = torch.tensor([1, 2, 3, 5, 6])
    assert bool((ko.cpu()[kept] == 5).all()) and bool((vo.cpu()[kept] == 5).all())
    if store == "bf16":
        assert torch.equal(ko[[0, 4]], k[[0, 4]])


def test_rows_without_ids_and_shared_pages(R):
    """Row i of sequence i; two sequences that share their first page read the same rows."""
    P = Pages(R, "int8", 2, 128, 16, [40, 40, 40])
    P.table[1, 0] = P.table[0, 0]
    for i in range(3):
        P.put(R, i, randn(10 + i, 40, 2, 128), randn(20 + i, 40, 2, 128))
    pos = torch.tensor([7, 7, 39], dtype=torch.int32, device="cuda")
    ko, vo = (torch.empty(3, 2, 128, device="cuda") for _ in range(2))
    R.riftkv_read(P.cache, P.table, pos, ko, vo, P.status)
    torch.cuda.synchronize()
    assert int(P.status) == 0 and torch.equal(ko[0], ko[1]) and torch.equal(vo[0], vo[1])
    assert torch.equal(ko[2].double().cpu(), P.rows(2, 40)[0][39])


# ----------------------------------------------------------------------------- attention
def attention(R, P, q, lens, table=None, scale=None, out=None, ws=None, stream=None):
    table = P.table if table is None else table
    out = torch.full_like(q, 77.0) if out is None else out
    if ws is None:
        size = R.riftkv_attention_workspace_size(P.cache, q.shape[0], q.shape[1], table.shape[1])
        ws = torch.full((size,), 0xAB, dtype=torch.uint8, device="cuda")
    R.riftkv_attention(P.cache, q, table, lens, out, ws, P.status, scale=scale, stream=stream)
    return out


def filled(R, store, n_kv, hd, page, lens, seed=0, k_scale=1.0, dtype=torch.bfloat16):
    P = Pages(R, store, n_kv, hd, page, lens, seed=seed)
    for i, n in enumerate(lens):
        P.put(R, i, randn(100 * seed + 2 * i, n, n_kv, hd, dtype=dtype, scale=k_scale),
              randn(100 * seed + 2 * i + 1, n, n_kv, hd, dtype=dtype))
    return P


def check(P, q, out, lens, scale=None, half=None):
    scale = q.shape[-1] ** -0.5 if scale is None else scale
    half = half_step(q.dtype) if half is None else half
    worst = 0.0
    for i, n in enumerate(lens):
        k, v = P.rows(i, n)
        ref, err = attend(q[i].double().cpu(), k, v, scale)
        got = out[i].double().cpu()
        # weights of bf16 queries are split in two bf16 terms: 2^-16 of each
        bound = err * (1 + 1e-3) + half * ref.abs() * (1 + 1e-3) + 1e-30
        if q.dtype == torch.bfloat16 and n:
            w = torch.softmax((k.repeat_interleave(q.shape[1] // k.shape[1], 1).transpose(0, 1) @ q[i].double().cpu()[:, :, None])[..., 0] * scale, -1)
            bound = bound + 2.0 ** -16 * (w[:, None] @ v.repeat_interleave(q.shape[1] // k.shape[1], 1).transpose(0, 1).abs())[:, 0]
        worst = max(worst, float(((got - ref).abs() / bound).max()))
    assert worst <= 1.0, worst


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 129, 300]


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "bf16"),
                                       ("f32", "fp8"), ("f32", "int8")])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv, group, page", [(2, 1, 16), (3, 4, 64), (1, 7, 32), (2, 16, 16), (1, 20, 128)])
def test_attention(R, dt, store, hd, n_kv, group, page):
    """Lengths around a tile and a page, in pages whose other bytes are NaN."""
    P = filled(R, store, n_kv, hd, page, LENS, seed=group, dtype=TYPES[dt])
    q = randn(5, len(LENS), n_kv * group, hd, dtype=TYPES[dt], scale=2)
    out = attention(R, P, q, torch.tensor(LENS, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(P.status) == 0
    check(P, q, out, LENS)


@pytest.mark.parametrize("store, n_kv, group, lens", [("bf16", 8, 4, [5001]), ("fp8", 2, 8, [9000, 1, 700]), ("int8", 1, 1, [4097, 4095]),
                                                      ("bf16", 1, 3, [17] * 300), ("fp8", 4, 2, list(range(0, 600, 5))),
                                                      ("bf16", 32, 1, [643, 355, 211, 131])])
@pytest.mark.parametrize("hd", [64, 128])
def test_attention_split_over_the_length(R, store, n_kv, group, lens, hd):
    """Few long sequences, many short ones, and both: the same bits from two calls."""
    P = filled(R, store, n_kv, hd, 32, lens, seed=3)
    q = randn(6, len(lens), n_kv * group, hd, scale=2)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = attention(R, P, q, n)
    again = attention(R, P, q, n)
    torch.cuda.synchronize()
    assert int(P.status) == 0 and torch.equal(out, again)
    check(P, q, out, lens)


def test_attention_sharp_and_flat(R):
    """Scores of hundreds (one key takes all) and a scale of zero (the mean of the values)."""
    lens = [200, 333]
    P = filled(R, "bf16", 2, 128, 16, lens, k_scale=30.0)
    q = randn(9, 2, 4, 128, scale=10)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    check(P, q, attention(R, P, q, n), lens)
    check(P, q, attention(R, P, q, n, scale=0.0), lens, scale=0.0)
    check(P, q, attention(R, P, q, n, scale=-0.05), lens, scale=-0.05)


def test_attention_of_strided_rows(R):
    lens = [40, 0, 90]
    P = filled(R, "fp8", 2, 64, 16, lens)
    wide = randn(4, 3, 1000)
    q = wide[:, 8:8 + 4 * 64].view(3, 4, 64)
    o = torch.full((3, 600), 5.0, dtype=torch.bfloat16, device="cuda")
    out = o[:, 16:16 + 4 * 64].view(3, 4, 64)
    attention(R, P, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), out=out)
    torch.cuda.synchronize()
    check(P, q, out, lens)
    assert bool((o[:, :16] == 5).all()) and bool((o[:, 16 + 4 * 64:] == 5).all())


@pytest.mark.parametrize("store", ["bf16", "int8", "f32"])
def test_attention_lengths_and_pages_out_of_range(R, store):
    """Their outputs are NaN and the status set; the others' are right."""
    dt = "f32" if store == "f32" else "bf16"
    lens = [50, 50, 50, 50, 50]
    P = filled(R, store, 2, 128, 16, lens, dtype=TYPES[dt])
    table = P.table.clone()
    table[1, 2] = -1
    table[3, 0] = P.k.shape[0]
    q = randn(5, 5, 4, 128, dtype=TYPES[dt])
    n = torch.tensor([50, 50, -3, 50, 65], dtype=torch.int32, device="cuda")     # 4 pages of 16 hold 64
    out = attention(R, P, q, n, table=table)
    torch.cuda.synchronize()
    assert int(P.status) == 2
    assert bool(torch.isnan(out[1:]).all())
    check(P, q[:1], out[:1], lens[:1])
    # past the length nothing is read: neither the entry nor the page
    P.status.zero_()
    n = torch.tensor([50, 32, 0, 0, 50], dtype=torch.int32, device="cuda")
    out = attention(R, P, q, n, table=table)
    torch.cuda.synchronize()
    assert int(P.status) == 0 and bool((out[2:4] == 0).all())
    check(P, q[:2], out[:2], [50, 32])


def test_attention_of_keys_and_values_that_are_not_finite(R):
    """They follow the formula: a key of NaN spoils its head, an infinite score of the
    negative sign has no weight, a value of NaN spoils its column."""
    n = 70
    P = Pages(R, "bf16", 2, 64, 16, [n] * 5)
    k, v = randn(1, n, 2, 64), randn(2, n, 2, 64)
    q = randn(3, 5, 2, 64).abs()          # positive: an infinite key of one sign gives an infinite score
    cases = [(k.clone(), v.clone()) for _ in range(5)]
    cases[0][0][20, 0, 7] = math.nan
    cases[1][0][33, 1] = -math.inf
    cases[2][1][69, 0, 5] = math.nan
    cases[3][0][2, 0] = math.inf
    cases[4][0][:, 1] = -math.inf         # every score of the head
    for i, (a, b) in enumerate(cases):
        P.put(R, i, a, b)
    lens = torch.full((5,), n, dtype=torch.int32, device="cuda")
    out = attention(R, P, q, lens).cpu()
    assert int(P.status) == 0
    nan = torch.isnan(out)
    want = torch.zeros_like(nan)
    want[0, 0] = True
    want[2, 0, 5] = True
    want[3, 0] = True
    want[4, 1] = True
    assert torch.equal(nan, want)
    kk, vv = cases[1][0].double().cpu(), v.double().cpu()
    for h in range(2):   # head 1 without the key
        keep = torch.arange(n) != (33 if h == 1 else -1)
        ref, err = attend(q[1, h:h + 1].double().cpu(), kk[keep, h:h + 1], vv[keep, h:h + 1], 64 ** -0.5)
        assert bool(((out[1, h:h + 1].double() - ref).abs() <= err + 2.0 ** -8 * ref.abs() * 1.001 + 2.0 ** -15).all())


@pytest.mark.parametrize("store", ["fp8", "int8"])
def test_attention_of_rows_that_could_not_be_quantised(R, store):
    n = 40
    P = Pages(R, store, 1, 128, 16, [n, n, n])
    k, v = randn(1, n, 1, 128), randn(2, n, 1, 128)
    bad = k.clone()
    bad[30, 0, 4] = math.inf
    P.put(R, 0, k, v)
    P.put(R, 1, bad, v)
    P.put(R, 2, k, bad)
    q = randn(3, 3, 2, 128)
    out = attention(R, P, q, torch.full((3,), n, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    check(P, q[:1], out[:1], [n])
    assert bool(torch.isnan(out[1:]).all())


def test_attention_wide_tables_and_no_pages(R):
    """A table far wider than the sequences, one with no columns, a batch of nothing."""
    lens = [33, 0, 5]
    P = filled(R, "bf16", 4, 64, 16, lens)
    table = torch.full((3, 4000), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, :P.table.shape[1]] = P.table
    q = randn(2, 3, 4, 64)
    out = attention(R, P, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), table=table)
    check(P, q, out, lens)
    out = attention(R, P, q, torch.zeros(3, dtype=torch.int32, device="cuda"), table=table[:, :0].contiguous())
    assert bool((out == 0).all())
    attention(R, P, q[:0], torch.zeros(0, dtype=torch.int32, device="cuda"), table=table[:0].contiguous())
    torch.cuda.synchronize()
    assert int(P.status) == 0


# ----------------------------------------------------------------------------- together
@pytest.mark.parametrize("store", ["bf16", "fp8", "int8"])
def test_decode_steps_in_a_graph(R, store):
    """rope, write and attention of one layer as a captured graph, replayed for several steps on another stream
    with the program's own work between, against the same calls made one by one and float64."""
    n_kv, group, hd, page, steps = 2, 3, 128, 16, 5
    lens = [14, 0, 47, 3]
    n = len(lens)
    cap = [x + steps for x in lens]
    dev = [Pages(R, store, n_kv, hd, page, cap) for _ in range(2)]
    for P in dev:
        for i, x in enumerate(lens):
            P.put(R, i, randn(i, x, n_kv, hd), randn(50 + i, x, n_kv, hd))
    freqs, mag = R.riftkv_rope_freqs(64, scaling="ramp", factor=4.0, original_len=4096, low=1, high=32)
    H = n_kv * group
    new = [randn(200 + t, n, (H + 2 * n_kv) * hd) for t in range(steps)]
    qkv, pos = torch.empty_like(new[0]), torch.tensor(lens, dtype=torch.int32, device="cuda")
    count = pos + 1
    q = qkv[:, :H * hd].view(n, H, hd)
    k = qkv[:, H * hd:(H + n_kv) * hd].view(n, n_kv, hd)
    v = qkv[:, (H + n_kv) * hd:].view(n, n_kv, hd)
    out = torch.empty(n, H, hd, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(R.riftkv_attention_workspace_size(dev[0].cache, n, H, dev[0].table.shape[1]), dtype=torch.uint8, device="cuda")

    def step(P):
        R.riftkv_rope(q, k, pos, freqs, layout="interleaved", magnitude=mag)
        R.riftkv_write(P.cache, k, v, P.table, pos, P.status)
        R.riftkv_attention(P.cache, q, P.table, count, out, ws, P.status)

    qkv.copy_(new[0])
    step(dev[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(dev[0])
    side = torch.cuda.Stream()
    for t in range(steps):
        qkv.copy_(new[t])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        got = out.clone()
        qq = q.clone()
        qkv.copy_(new[t])
        out.zero_()
        step(dev[1])
        torch.cuda.synchronize()
        assert torch.equal(out, got), t
        check(dev[1], qq, out, count.tolist())
        pos += 1
        count += 1
    assert int(dev[0].status) == 0 and int(dev[1].status) == 0
    for a, b in ((dev[0].k, dev[1].k), (dev[0].v, dev[1].v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_offsets_past_32_bits(R):
    """Pages at the end of a pool whose arrays pass 4 GB (2^32 bytes, 2^31 values): written, read and attended to."""
    n_pages, n_kv, page, hd = 140_000, 8, 16, 128
    k = torch.empty(n_pages, n_kv, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 31
    cache = R.riftkv_cache(k, v)
    n = 100
    table = torch.arange(n_pages - 1, n_pages - 1 - 7, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    a, b = randn(1, n, n_kv, hd), randn(2, n, n_kv, hd)
    R.riftkv_write(cache, a, b, table, pos, status, seq_ids=ids)
    ko, vo = torch.empty_like(a), torch.empty_like(b)
    R.riftkv_read(cache, table, pos, ko, vo, status, seq_ids=ids)
    q = randn(3, 1, 32, hd)
    out = torch.empty_like(q)
    ws = torch.empty(R.riftkv_attention_workspace_size(cache, 1, 32, 7), dtype=torch.uint8, device="cuda")
    R.riftkv_attention(cache, q, table, torch.tensor([n], dtype=torch.int32, device="cuda"), out, ws, status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(ko, a) and torch.equal(vo, b)
    assert torch.equal(k[n_pages - 1, :, 3], a[3]) and torch.equal(v[n_pages - 7, :, 2], b[98])
    ref, err = attend(q[0].double().cpu(), a.double().cpu(), b.double().cpu(), hd ** -0.5)
    got = out[0].double().cpu()
    # (weights in two bf16 terms: 2^-16 of each, of values up to 5)
    assert bool(((got - ref).abs() <= err + 2.0 ** -8 * ref.abs() * 1.001 + 2.0 ** -16 * 5).all())


def test_calls_on_two_streams_at_once(R):
    """Each with its own workspace and outputs, over the same pages: as one after the other."""
    lens = [3000, 17, 900]
    P = filled(R, "fp8", 2, 128, 16, lens)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qs = [randn(40 + i, 3, 2 * g, 128) for i, g in enumerate((4, 16))]
    size = [R.riftkv_attention_workspace_size(P.cache, 3, q.shape[1], P.table.shape[1]) for q in qs]
    want = [attention(R, P, q, n) for q in qs]
    ws = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in size]
    outs = [torch.empty_like(q) for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, o, w, st in zip(qs, outs, ws, streams):
            attention(R, P, q, n, out=o, ws=w, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs)) and int(P.status) == 0


@pytest.mark.parametrize("store, dt, group, lens", [("bf16", "bf16", 16, [5000, 70]), ("int8", "f32", 16, [2100] * 3),
                                                    ("f32", "f32", 17, [40, 1500]), ("fp8", "bf16", 40, [64] * 40)])
def test_attention_in_a_graph(R, store, dt, group, lens):
    """Large groups (more than 64 KB of LDS), captured and replayed with lengths that change between replays."""
    P = filled(R, store, 1, 128, 16, lens, dtype=TYPES[dt])
    q = randn(7, len(lens), group, 128, dtype=TYPES[dt])
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(R.riftkv_attention_workspace_size(P.cache, len(lens), group, P.table.shape[1]), dtype=torch.uint8, device="cuda")
    attention(R, P, q, n, out=out, ws=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attention(R, P, q, n, out=out, ws=ws)
    for cut in (0, 1, 33, 0):
        n.copy_(torch.tensor([max(0, x - cut) for x in lens], dtype=torch.int32))
        out.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        check(P, q, out, [max(0, x - cut) for x in lens])
        assert torch.equal(out, attention(R, P, q, n))
    assert int(P.status) == 0


def test_refusals_leave_the_outputs(R):
    P = filled(R, "bf16", 2, 64, 16, [20])
    q = randn(2, 1, 4, 64)
    n = torch.tensor([20], dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 5)
    ws = torch.empty(R.riftkv_attention_workspace_size(P.cache, 1, 4, P.table.shape[1]), dtype=torch.uint8, device="cuda")
    for args in ((q.float(), P.table, n, out), (q, P.table.long(), n, out), (q, P.table, n.long(), out),
                 (q[:, :3], P.table, n, out[:, :3]), (q, P.table, n, out[..., :32]), (q.cpu(), P.table, n, out)):
        with pytest.raises((TypeError, ValueError, R.RiftError)):
            R.riftkv_attention(P.cache, *args, ws, P.status)
    with pytest.raises(R.RiftError) as e:
        R.riftkv_attention(P.cache, q, P.table, n, out, ws[:0], P.status)
    with pytest.raises(TypeError):
        R.riftkv_cache(P.k.half(), P.v.half())
    with pytest.raises(ValueError):
        R.riftkv_cache(P.k, P.v[:1])
    with pytest.raises(ValueError):
        R.riftkv_cache(P.k.view(torch.int8)[..., :64].contiguous(), P.v.view(torch.int8)[..., :64].contiguous())
    torch.cuda.synchronize()
    assert bool((out == 5).all()) and int(P.status) == 0
