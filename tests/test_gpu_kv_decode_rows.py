"""What a decode step over pages writes: the new token's keys and values against float64, every other byte as it was."""
import numpy as np
import pytest
import torch

import synth
from oracle import rift_oracle as O
from tests.kv_testlib import LARGEST, half_step
from tests.rift_testlib import f64, oracle_layer_weights
from tests.test_gpu_kv_decode import Run

pytestmark = pytest.mark.gpu

WHOLE = synth.ModelShape(d=1280, n_heads=10, head_dim=128, ffn=2560, n_layers=2)    # rows through riftkv_write's kernel
SPLIT = synth.ModelShape(d=1024, n_heads=8, head_dim=128, ffn=2048, n_layers=2)     # sums, rotation and pages in one kernel
SPLIT64 = synth.ModelShape(d=2048, n_heads=32, head_dim=64, ffn=2048, n_layers=2)


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def new_rows(x, W, m, positions):
    """float64 keys and values [n][heads][hd] of the new tokens, and how far a step may be from them before they are
    stored: the normalised row is float32 (its mean of squares and root 2^-18 at most), rounded to bf16; d products summed in
    float32; the rotation's sines, products and sum 4 steps of float32; rounded to bf16."""
    half = half_step(torch.bfloat16)
    h = O.rmsnorm(x, W["g_attn"], m.rms_eps)
    out = []
    for name in ("wk", "wv"):
        y = (h @ W[name].T).reshape(-1, m.n_heads, m.head_dim)
        e = (np.abs(h) @ np.abs(W[name]).T).reshape(y.shape) * (half + 2.0 ** -18 + m.d * 2.0 ** -24)
        if name == "wk":
            y = O.rope(y, positions, m.rope_base)
            # an element's error after the rotation is at most its own and its partner's
            e = e + np.roll(e, m.head_dim // 2, axis=-1)
            e = e + (np.abs(y) + np.abs(np.roll(y, m.head_dim // 2, axis=-1))) * 4 * 2.0 ** -23
        out.append((y, e + half * (np.abs(y) + e)))
    return out


def byte_of(most, dtype):
    """The smallest b >= 1 with most <= largest * 2^(b - 127), of float64 magnitudes."""
    b = np.ceil(np.log2(np.maximum(most, 1e-300) / LARGEST[dtype])).astype(np.int64) + 127
    b += most > LARGEST[dtype] * 2.0 ** (b - 127.0)
    b -= most <= LARGEST[dtype] * 2.0 ** (b - 128.0)
    return np.maximum(b, 1)


@pytest.mark.parametrize("pages_of", ["bf16", "fp8", "int8"])
@pytest.mark.parametrize("m", [WHOLE, SPLIT, SPLIT64], ids=["whole128", "split128", "split64"])
@pytest.mark.parametrize("lens, page", [([30, 7, 64, 1, 15], 16), ([100], 32)])
def test_new_rows(R, m, pages_of, lens, page):
    n = len(lens)
    r = Run(R, m, 2, lens, pages_of, page=page, padding=1)
    W = oracle_layer_weights(r.W[0], "bf16")
    c = r.cache
    arrays = [a for a in (c.k, c.v, c.k_scale, c.v_scale) if a is not None]
    for t in range(2):
        before = [a.view(torch.uint8).clone() for a in arrays]
        r.step(t)
        torch.cuda.synchronize()
        assert int(r.status) == 0
        at = np.array([L + t for L in lens])
        page_of = r.table[torch.arange(n).cuda(), torch.from_numpy(at // page).cuda()].long()
        row = torch.from_numpy(at % page).cuda()
        # the new rows' bytes changed, in every layer, and no others
        for a, b in zip(arrays, before):
            same = a.view(torch.uint8) == b
            same = same.all(-1) if a.dim() == 5 else same     # [layers][pages][heads][page]
            for i, j in zip(page_of.tolist(), row.tolist()):
                assert a.dim() == 4 or not bool(same[:, i, :, j].any())
                same[:, i, :, j] = True
            assert bool(same.all())
        for name, (y, bound) in zip(("k", "v"), new_rows(f64(r.new[t], "bf16")[:n], W, m, at)):
            pages, scales = getattr(c, name), getattr(c, name + "_scale")
            got = pages[0].view(torch.uint8)[page_of, :, row].cpu().view(pages.dtype).to(torch.float32).double().numpy()
            if scales is not None:
                byte = scales[0][page_of, :, row].cpu().long().numpy()
                most, e = np.abs(y).max(-1), bound.max(-1)
                lo, hi = byte_of(np.maximum(np.abs(y) - bound, 0).max(-1), pages.dtype), byte_of(most + e, pages.dtype)
                assert ((byte >= lo) & (byte <= hi)).all(), (name, byte, lo, hi)
                scale = 2.0 ** (byte - 127.0)[..., None]
                got = got * scale
                # a code is off by half a step: e4m3 relative, or of its smallest numbers 2^-10; int8 1/2
                half = np.maximum(half_step(pages.dtype) * np.abs(got), 2.0 ** -10 * scale) if pages_of == "fp8" else scale / 2
                bound = bound + half
            worst = (np.abs(got - y) / bound).max()
            assert worst <= 1.0, (t, name, worst)
