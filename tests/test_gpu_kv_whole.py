"""Attention over heads that one workgroup takes whole, with each number of waves, and
over those just too long for it."""
import pytest
import torch

from tests.test_gpu_kv import TYPES, attention, check, filled, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "int8")])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("n_kv, group, lens", [(1, 8, [512, 0, 385, 511]), (3, 1, [400, 768, 1, 33]), (16, 2, [1024, 390, 17, 640, 0, 993]),
                                               (2, 16, [417, 480]), (1, 20, [500, 31]), (64, 1, [130, 384, 60, 500]),
                                               (96, 1, [1056]), (2, 3, [240, 256, 7]), (128, 1, [300, 352, 2])])
def test_heads_whole_or_nearly(R, dt, store, hd, n_kv, group, lens):
    """Ragged lengths up to the table's width, the same bits from two calls."""
    P = filled(R, store, n_kv, hd, 32, lens, seed=n_kv, dtype=TYPES[dt])
    q = randn(7, len(lens), n_kv * group, hd, dtype=TYPES[dt], scale=2)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = attention(R, P, q, n)
    again = attention(R, P, q, n)
    torch.cuda.synchronize()
    assert int(P.status) == 0 and torch.equal(out, again)
    check(P, q, out, lens)


@pytest.mark.parametrize("store", ["bf16", "fp8"])
def test_a_whole_head_in_a_graph(R, store):
    """Replayed with other lengths, the table's whole width and none among them."""
    lens = [450, 512, 20]
    P = filled(R, store, 2, 128, 16, [512] * 3, seed=11)
    q = randn(8, 3, 32, 128, scale=2)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.zeros(R.riftkv_attention_workspace_size(P.cache, 3, 32, P.table.shape[1]), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    R.riftkv_attention(P.cache, q, P.table, n, out, ws, P.status)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        R.riftkv_attention(P.cache, q, P.table, n, out, ws, P.status)
    for lens in ([450, 512, 20], [0, 1, 512], [511, 0, 33]):
        n.copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(5)
        ws.random_(0, 255)
        g.replay()
        torch.cuda.synchronize()
        check(P, q, out, lens)
    assert int(P.status) == 0


@pytest.mark.parametrize("store", ["bf16", "int8"])
@pytest.mark.parametrize("page, hd, lens", [(4096, 64, [4096, 1, 4097, 0, 4095]), (1024, 128, [1025, 3000, 1024])])
def test_large_pages(R, store, page, hd, lens):
    P = filled(R, store, 2, hd, page, lens, seed=21)
    q = randn(9, len(lens), 6, hd, scale=2)
    out = attention(R, P, q, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(P.status) == 0
    check(P, q, out, lens)


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("n_kv, group, n, long", [(1, 3, 257, {200: 3000}), (2, 1, 700, {0: 1500, 350: 1, 699: 2049}), (1, 18, 300, {299: 1300}),
                                                  (1, 2, 1030, {})])
def test_more_sequences_than_a_wave_holds(R, dt, store, n_kv, group, n, long):
    """Split heads of many ragged sequences, most short, many without tokens."""
    lens = [(7 * i) % 40 if i % 3 else 0 for i in range(n)]
    for i, x in long.items():
        lens[i] = x
    room = lens if long else [1100] + lens[1:]     # a wide table all the same
    P = filled(R, store, n_kv, 64, 16, room, seed=31, dtype=TYPES[dt])
    q = randn(10, n, n_kv * group, 64, dtype=TYPES[dt], scale=2)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = attention(R, P, q, t)
    again = attention(R, P, q, t)
    torch.cuda.synchronize()
    assert int(P.status) == 0 and torch.equal(out, again)
    check(P, q, out, lens)


def test_many_sequences_none_with_tokens(R):
    P = filled(R, "bf16", 1, 64, 16, [1100] + [1] * 299, seed=32)
    q = randn(12, 300, 2, 64)
    out = attention(R, P, q, torch.zeros(300, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(P.status) == 0 and not bool(out.any())
