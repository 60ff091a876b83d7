"""Every tensor argument of the paged cache's calls, wrong in each way that a call can see
before it launches anything: refused by name, with nothing written."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def calls(R, n, heads):
    """(function, arguments, names of the tensors, those that are rows) of each call, for n rows."""
    dev, hd = "cuda", 64
    k = torch.zeros(4, heads, 16, hd, device=dev, dtype=torch.bfloat16)
    cache = R.riftkv_cache(k, torch.zeros_like(k))
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)
    rows = lambda h: torch.ones(n, h, hd, dtype=torch.bfloat16, device=dev)
    ws = torch.zeros(R.riftkv_attention_workspace_size(cache, n, 2 * heads, 2), dtype=torch.uint8, device=dev)
    freqs, _ = R.riftkv_rope_freqs(32)
    place = dict(page_table=i32(n, 2), positions=i32(n), status=i32(1), seq_ids=i32(n))
    return [(lambda a: R.riftkv_write(cache, **a), dict(k=rows(heads), v=rows(heads), **place), ("k", "v"), ()),
            (lambda a: R.riftkv_read(cache, **a), dict(k_out=rows(heads), v_out=rows(heads), **place), ("k_out", "v_out"), ("k_out", "v_out")),
            (lambda a: R.riftkv_attention(cache, **a),
             dict(q=rows(2 * heads), page_table=i32(n, 2), lens=i32(n) + 1, out=rows(2 * heads), workspace=ws, status=i32(1)), ("q", "out"), ("out",)),
            (lambda a: R.riftkv_rope(freqs=freqs, **a),
             dict(q=rows(heads), k=rows(heads), positions=i32(n), q_out=rows(heads), k_out=rows(heads)), ("q", "k", "q_out", "k_out"), ("q_out", "k_out"))], cache


@pytest.mark.parametrize("n, heads", [(1, 2), (3, 2), (1, 1), (5, 1)])
def test_each_argument(R, n, heads):
    made, cache = calls(R, n, heads)
    for call, args, rows, outs in made:
        for name, t in args.items():
            wrong = {"type": t.to(torch.float16 if t.dtype == torch.bfloat16 else torch.int64), "host": t.cpu()}
            if name != "workspace":
                wrong["longer"] = torch.cat([t, t])
            if name in rows and heads > 1:
                wrong["heads apart"] = torch.cat([t, t], 2)[:, :, :64]
                wrong["transposed"] = t.transpose(1, 2).contiguous().transpose(1, 2)
            elif name not in rows and name != "status" and t.numel() > 1:
                wrong["strided"] = torch.stack([t, t], -1)[..., 0]
            for how, bad in wrong.items():
                if name == "page_table" and how == "longer":     # more sequences are right for rows with their own numbers
                    if "seq_ids" in args:
                        continue
                with pytest.raises((TypeError, ValueError)):
                    call({**args, name: bad})
                    pytest.fail(f"{name}: {how}")
        torch.cuda.synchronize()
        assert all(bool((args[o] == 1).all()) for o in outs)
    assert not bool(cache.k.any())


@pytest.mark.parametrize("heads", [1, 3])
def test_strides_of_one_row_do_not_matter(R, heads):
    """A single row, or a single head, of a tensor of any stride."""
    hd = 64
    g = torch.Generator().manual_seed(4)
    k = torch.zeros(2, heads, 16, hd, device="cuda", dtype=torch.bfloat16)
    cache = R.riftkv_cache(k, torch.zeros_like(k))
    table = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    pos, status = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    row = torch.randn(heads, hd, generator=g).bfloat16().cuda()
    for odd in (row.view(1, heads, hd), row.as_strided((1, heads, hd), (3, hd, 1)), row.as_strided((1, heads, hd), (0, hd, 1))):
        cache.k.zero_()
        R.riftkv_write(cache, odd, odd, table, pos, status)
        back = torch.zeros(8, heads, hd, device="cuda", dtype=torch.bfloat16)[5:6]
        R.riftkv_read(cache, table, pos, back, torch.zeros_like(back), status)
        assert torch.equal(back[0], row) and torch.equal(cache.k[1, :, 0], row)
    if heads == 1:
        many = torch.randn(3, 2, hd, generator=g).bfloat16().cuda()[:, 1:]      # one head, two heads' width apart
        ids = torch.zeros(3, dtype=torch.int32, device="cuda")
        R.riftkv_write(cache, many, many, table, torch.arange(3, dtype=torch.int32, device="cuda"), status, seq_ids=ids)
        assert torch.equal(cache.k[1, 0, :3], many[:, 0])
    assert int(status) == 0
