"""Calls of the paged key-value cache of more rows than one launch has threads for (2^32)."""
import numpy as np
import pytest
import torch

from tests.kv_testlib import Pages, attend, half_step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    yield R
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows, nq, nk, hd, rot, layout", [((1 << 24) + 3, 1, 0, 16, 16, "half"), ((1 << 24) + 300, 0, 1, 16, 16, "interleaved"),
                                                           ((1 << 26) // 3 + 5, 2, 1, 2, 2, "half")])
def test_rope_of_many_rows(R, rows, nq, nk, hd, rot, layout):
    """All rows at once are what their parts are."""
    torch.manual_seed(1)
    x = torch.randn(rows, (nq + nk) * hd, device="cuda", dtype=torch.bfloat16)
    q, k = (x[:, a * hd:b * hd].view(rows, b - a, hd) if b > a else None for a, b in ((0, nq), (nq, nq + nk)))
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (rows,), dtype=torch.int32, device="cuda")
    freqs, mag = R.riftkv_rope_freqs(rot)
    outs = [None if t is None else torch.zeros(t.shape, dtype=t.dtype, device="cuda") for t in (q, k)]
    parts = [None if t is None else torch.zeros(t.shape, dtype=t.dtype, device="cuda") for t in (q, k)]
    R.riftkv_rope(q, k, pos, freqs, *outs, layout=layout, magnitude=mag)
    step = rows // 3
    for a in range(0, rows, step):
        cut = lambda t: None if t is None else t[a:a + step]
        R.riftkv_rope(cut(q), cut(k), pos[a:a + step], freqs, cut(parts[0]), cut(parts[1]), layout=layout, magnitude=mag)
    for a, b in zip(outs, parts):
        assert a is None or torch.equal(a, b)
        assert a is None or not bool((b[-1] == 0).all())


def test_rows_of_many_launches(R):
    """Rows around the ends of launches go to their places, and come back; the others are padding."""
    hd, page = 64, 16
    P = Pages(R, "bf16", 1, hd, page, [200])
    for rows, name in (((1 << 27) + 9, "write"), ((1 << 28) + 17, "read")):
        data = torch.zeros(rows, 1, hd, device="cuda", dtype=torch.bfloat16)
        pos = torch.full((rows,), -1, device="cuda", dtype=torch.int32)
        ids = torch.zeros(rows, device="cuda", dtype=torch.int32)
        at = torch.tensor([0, 1, 77, rows // 2, *range(rows - 40, rows)], device="cuda")
        pos[at] = torch.arange(at.numel(), device="cuda", dtype=torch.int32)
        if name == "write":
            want = torch.randn(at.numel(), 1, hd, generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
            data[at] = want
            R.riftkv_write(P.cache, data, data, P.table, pos, P.status, seq_ids=ids)
            k, v = P.rows(0, at.numel())
            assert torch.equal(k, want.double().cpu()) and torch.equal(v, k)
            assert bool(torch.isnan(P.rows(0, 200)[0][at.numel():]).all())   # nothing else was written
        else:
            R.riftkv_read(P.cache, P.table, pos, data, data, P.status, seq_ids=ids)
            assert torch.equal(data[at], want)
            data[at] = 0
            assert not bool(data.view(torch.int32).any())
        del data, pos, ids
    assert int(P.status) == 0


def test_attention_of_many_heads(R):
    """More heads than a launch of four waves each holds: sequences of one token (their value),
    of none, and some as long as the table."""
    n_seq, n_kv, hd, page, wide, pool = 65535, 257, 64, 16, 33, 40
    torch.manual_seed(2)
    k = torch.randn(pool, n_kv, page, hd, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(pool, n_kv, page, hd, device="cuda", dtype=torch.bfloat16)
    cache = R.riftkv_cache(k, v)
    table = torch.randint(0, pool, (n_seq, wide), device="cuda", dtype=torch.int32)
    lens = torch.ones(n_seq, device="cuda", dtype=torch.int32)
    lens[5::7] = 0
    long = {0: 528, 1: 33, 30000: 512, n_seq - 2: 17, n_seq - 1: 527}
    for i, n in long.items():
        lens[i] = n
    q = torch.randn(n_seq, n_kv, hd, device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(R.riftkv_attention_workspace_size(cache, n_seq, n_kv, wide), dtype=torch.uint8, device="cuda")
    R.riftkv_attention(cache, q, table, lens, out, ws, status)
    assert int(status) == 0
    one = lens == 1
    assert torch.equal(out[one], v[:, :, 0][table[:, 0].long()][one])
    assert not bool(out[lens == 0].any())
    for i, n in long.items():
        pages = table[i].long()
        kk, vv = (x[pages].transpose(1, 2).flatten(0, 1)[:n].double().cpu() for x in (k, v))
        ref, err = attend(q[i].double().cpu(), kk, vv, hd ** -0.5)
        got = out[i].double().cpu()
        assert bool(((got - ref).abs() <= half_step(torch.bfloat16) * ref.abs() + 1.01 * err).all())


def test_frequencies_of_another_byte_order(R):
    freqs, _ = R.riftkv_rope_freqs(16)
    x = torch.zeros(1, 1, 16, device="cuda", dtype=torch.bfloat16)
    pos = torch.zeros(1, device="cuda", dtype=torch.int32)
    with pytest.raises(TypeError):
        R.riftkv_rope(x, None, pos, freqs.astype(">f8"))
    assert np.dtype(">f8").char == freqs.dtype.char
