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
