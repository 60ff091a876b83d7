"""Attention's weights keep their 24 bits on the way into the second product, whatever the pages hold."""

import pytest
import torch

from tests.kv_testlib import LARGEST, Pages, attend, half_step, quantise
from tests.test_gpu_kv import TYPES, attention, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def kept(x, store):
    """The values that rows x have once they are in pages."""
    if store not in LARGEST:
        return x.to(store).double()
    code, byte = quantise(x, store)
    return torch.ldexp(code, (byte - 127)[..., None].double())


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "fp8")])
@pytest.mark.parametrize("hd, seqs", [(64, 48), (128, 48), (128, 2)])
def test_values_that_cancel(R, dt, store, hd, seqs):
    """A token of weight 1 and value V, and J tokens of one weight p whose values add up to almost -V / p: what p is
    off by is left over, 2^-17 p of it where a weight is two bf16 numbers."""
    n_kv, J = 4, 3
    P = Pages(R, store, n_kv, hd, 16, [J + 1] * seqs, seed=hd)
    g = torch.Generator().manual_seed(7)
    scale = hd ** -0.5
    q = torch.zeros(seqs, n_kv, hd)
    q[..., 0] = 1.0
    key = torch.zeros(seqs, n_kv, hd)
    key[..., 0] = -(0.7 + 5.0 * torch.rand(seqs, n_kv, generator=g, dtype=torch.float64)).float()
    key = kept(key, P.store)                                    # as the pages hold it
    scale32 = float(torch.tensor(scale, dtype=torch.float32))
    s = key[..., 0] * scale32                                   # every other product is 0
    p = torch.exp(s)
    V = 0.5 + 0.5 * torch.rand(seqs, n_kv, hd, generator=g, dtype=torch.float64)
    V = V * torch.where(torch.rand(seqs, n_kv, hd, generator=g) < 0.5, -1.0, 1.0)
    V = kept(V.float(), P.store)
    rows, rest = [V], -V / p[..., None]
    for _ in range(J):
        rows.append(kept(rest.float(), P.store))
        rest = rest - rows[-1]
    dtype = TYPES[dt]
    for i in range(seqs):
        k = torch.stack([torch.zeros_like(key[i])] + [key[i]] * J)
        v = torch.stack([x[i] for x in rows])
        assert torch.equal(v.to(dtype).double(), v)
        P.put(R, i, k.to(dtype).cuda(), v.to(dtype).cuda())
    k0, v0 = P.rows(0, J + 1)
    assert torch.equal(v0, torch.stack([x[0] for x in rows])) and torch.equal(k0[1], key[0])
    out = attention(R, P, q.to(dtype).cuda(), torch.full((seqs,), J + 1, dtype=torch.int32, device="cuda"), scale=scale32)
    torch.cuda.synchronize()
    assert int(P.status) == 0
    total = 1 + J * p[..., None]
    ref = (V + p[..., None] * sum(rows[1:])) / total
    size = (V.abs() + p[..., None] * sum(x.abs() for x in rows[1:])) / total
    # an exponent: two products and the scale's log2(e), half a step each; its power of two a step; every term of every
    # weighted value added up in float32, a step each; the sum of the weights multiplies what is left only
    rel = s.abs()[..., None] * 3 * 2.0 ** -24 + 2.0 ** -23 + 3 * (J + 1) * 2.0 ** -23
    bound = rel * size + half_step(dtype) * ref.abs() * (1 + 2.0 ** -6)
    worst = float(((out.double().cpu() - ref).abs() / bound).max())
    assert worst <= 1.0, worst


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("store", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("exponent", [60, -60, -100, -106, -112, -118])
def test_values_of_any_size(R, dt, store, hd, exponent):
    """Values around 2^exponent.  With 8-bit pages a weight times its row's scale loses what is below 2^-133, of each
    token's code."""
    lens = [40, 200]
    P = Pages(R, store, 2, hd, 16, lens, seed=1)
    for i, n in enumerate(lens):
        v = torch.randn(n, 2, hd, generator=torch.Generator().manual_seed(50 + i)).double().mul(2.0 ** exponent)
        P.put(R, i, randn(i, n, 2, hd), v.to(torch.bfloat16).cuda())
    q = randn(5, 2, 8, hd, dtype=TYPES[dt], scale=2)
    out = attention(R, P, q, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(P.status) == 0
    for i, n in enumerate(lens):
        k, v = P.rows(i, n)
        x = q[i].double().cpu()
        ref, err = attend(x, k, v, hd ** -0.5)
        bound = err * (1 + 1e-3) + half_step(q.dtype) * ref.abs() * (1 + 1e-3) + 2.0 ** -149
        if P.store in LARGEST:
            page, row = P.table[i, torch.arange(n) // 16].long().cpu(), torch.arange(n) % 16
            codes = P.v.view(torch.uint8).cpu()[page, :, row].view(P.store).float().double().abs()    # [n][2][hd]
            s = (k.repeat_interleave(4, 1).transpose(0, 1) @ x[:, :, None])[..., 0] * hd ** -0.5      # [heads][n]
            total = torch.exp(s - s.amax(-1, keepdim=True)).sum(-1)
            bound = bound + 2.0 ** -133 * codes.sum(0).repeat_interleave(4, 0) / total[:, None]
        worst = float(((out[i].double().cpu() - ref).abs() / bound).max())
        assert worst <= 1.0, worst
