"""The calls for long contexts at their largest: more workgroups than one launch takes, places past 32 bits, the widest tables."""
import pytest
import torch

from tests.kv_ranges_testlib import attend, check, randn, selection

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    yield R
    torch.cuda.empty_cache()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def space(size):
    return torch.empty(max(256, size), dtype=torch.uint8, device="cuda")


def test_attentions_of_many_launches(R):
    """33,553,920 (sequence, key head) pairs: a token each, whose value is the output; some have none."""
    n, kv, hd = 65535, 512, 64
    k = torch.randn(4, kv, 16, hd, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(4, kv, 16, hd, device="cuda", dtype=torch.bfloat16)
    cache, status = R.riftkv_cache(k, v), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(n, kv, hd, device="cuda", dtype=torch.bfloat16)
    table = (torch.arange(n, device="cuda", dtype=torch.int32) % 4)[:, None].contiguous()
    lens = (torch.arange(n, device="cuda", dtype=torch.int32) % 3 != 0).int().contiguous()
    out = torch.full_like(q, 7.0)
    want = torch.where(lens[:, None, None] > 0, v[:, :, 0][table[:, 0].long()], torch.zeros((), dtype=torch.bfloat16, device="cuda"))
    ws = space(R.riftkv_attention_shared_workspace_size(cache, n, kv, 0, 1))
    R.riftkv_attention_shared(cache, q, table[0, :0], 0, table, lens, out, ws, status)
    assert torch.equal(out, want)
    out.fill_(7.0)
    lists = torch.zeros(n, kv, 1, device="cuda", dtype=torch.int32)
    ws = space(R.riftkv_attention_pages_workspace_size(cache, n, kv, 1))
    R.riftkv_attention_pages(cache, q, table, lens, lists, out, ws, status)
    assert torch.equal(out, want) and int(status) == 0


def test_selection_of_many_launches(R):
    """16,776,960 (sequence, key head) pairs of two pages, the better one of which is taken."""
    n, kv, hd = 65535, 256, 64
    k = torch.empty(8, kv, 16, hd, device="cuda", dtype=torch.bfloat16)
    cache, status = R.riftkv_cache(k, k), torch.zeros(1, dtype=torch.int32, device="cuda")
    bounds = torch.zeros(8, kv, 2, hd, device="cuda", dtype=torch.bfloat16)
    bounds[:, :, 1, 0] = torch.randn(8, kv, device="cuda", dtype=torch.bfloat16).abs()
    q = torch.zeros(n, kv, hd, device="cuda", dtype=torch.bfloat16)
    q[:, :, 0] = 1
    a = torch.arange(n, device="cuda", dtype=torch.int32)
    table = torch.stack((a % 8, (a // 8 + a + 1) % 8), 1).contiguous()
    lens = torch.full((n,), 32, device="cuda", dtype=torch.int32)
    pages = torch.full((n, kv, 1), -5, device="cuda", dtype=torch.int32)
    ws = space(R.riftkv_select_pages_workspace_size(cache, n, 2))
    R.riftkv_select_pages(cache, bounds, q, table, lens, pages, ws, status, keep_first=0, keep_last=0)
    score = bounds[:, :, 1, 0][table.long()]                  # [n][2][kv]
    assert torch.equal(pages[:, :, 0], (score[:, 1] > score[:, 0]).int()) and int(status) == 0


def test_places_past_32_bits(R):
    """Pages and bounds of more than 2^32 bytes and elements: the last pages of 40 GB are read where they are."""
    kv, hd, page, n_pages = 8, 128, 16, 1_250_000
    k = torch.zeros(n_pages, kv, page, hd, device="cuda", dtype=torch.bfloat16)
    assert k.numel() > 1 << 34
    cache, status = R.riftkv_cache(k, k), torch.zeros(1, dtype=torch.int32, device="cuda")
    at = [n_pages - 1, 3, n_pages - 70, 700_000, n_pages - 2]
    rows = randn(3, len(at), kv, page, hd)
    k[torch.tensor(at, device="cuda")] = rows
    table, lens = i32([at]), i32([16 * len(at) - 3])
    bounds = torch.full((n_pages, kv, 2, hd), 9.0, device="cuda", dtype=torch.bfloat16)
    R.riftkv_page_bounds(cache, bounds, table, lens, status)
    flat = rows.transpose(1, 2).flatten(0, 1)[:int(lens)]      # [tokens][kv][hd]
    for i, p in enumerate(at):
        x = flat[16 * i:16 * (i + 1)]
        assert torch.equal(bounds[p], torch.stack((x.amin(0), x.amax(0)), 1))
    assert int((bounds != 9.0).any(-1).any(-1).any(-1).sum()) == len(at)
    q = randn(4, 1, 2 * kv, hd, scale=2)
    lists = torch.empty(1, kv, 3, device="cuda", dtype=torch.int32)
    R.riftkv_select_pages(cache, bounds, q, table, lens, lists, space(R.riftkv_select_pages_workspace_size(cache, 1, 5)), status)
    assert torch.equal(lists.cpu(), selection(bounds[torch.tensor(at, device="cuda")], torch.arange(5)[None], q, [5], kv, 3, 1, 1))
    out = torch.empty_like(q)
    R.riftkv_attention_pages(cache, q, table, lens, lists, out, space(R.riftkv_attention_pages_workspace_size(cache, 1, 2 * kv, 3)), status)
    f, qd = flat.double().cpu(), q[0].double().cpu()
    for h in range(kv):
        tokens = [t for p in lists[0, h].tolist() for t in range(16 * p, min(16 * (p + 1), int(lens)))]
        o, e = attend(qd[2 * h:2 * h + 2], f[tokens, h:h + 1], f[tokens, h:h + 1], hd ** -0.5)
        check(out[0, 2 * h:2 * h + 2], o, e, q.dtype)
    for seqs, times in ((2, 1), (40, 10)):                     # a prefix walked, and by rows: the pages ten times over
        front = i32(at * times)
        n = 16 * len(at) * times - 3
        qs = randn(5, seqs, 2 * kv, hd, scale=2)
        none = torch.zeros(seqs, device="cuda", dtype=torch.int32)
        o = torch.empty_like(qs)
        R.riftkv_attention_shared(cache, qs, front, n, torch.empty(seqs, 0, device="cuda", dtype=torch.int32), none, o,
                                  space(R.riftkv_attention_shared_workspace_size(cache, seqs, 2 * kv, n, 0)), status)
        every = rows.transpose(1, 2).flatten(0, 1).repeat(times, 1, 1)[:n].double().cpu()
        for i in (0, seqs - 1):
            want, e = attend(qs[i].double().cpu(), every, every, hd ** -0.5)
            e = e + 2.0 ** -17 * attend(qs[i].double().cpu(), every, every.abs(), hd ** -0.5)[0]
            check(o[i], want, e, qs.dtype)
    assert int(status) == 0


@pytest.mark.parametrize("page, top", [(4096, 1 << 18), (16, 1 << 20)])
def test_the_longest_lists(R, page, top):
    """Lists of 2^30 tokens at most, all but a few places empty."""
    k = randn(1, 3, 1, page, 64)
    v = randn(2, 3, 1, page, 64)
    cache, status = R.riftkv_cache(k, v), torch.zeros(1, dtype=torch.int32, device="cuda")
    lists = torch.full((1, 1, top), -1, device="cuda", dtype=torch.int32)
    lists[0, 0, 0], lists[0, 0, top // 2], lists[0, 0, top - 1] = 2, 0, 1
    lens, table = i32([2 * page + 7]), i32([[0, 1, 2]])
    q = randn(3, 1, 2, 64, scale=2)
    out = torch.empty_like(q)
    R.riftkv_attention_pages(cache, q, table, lens, lists, out, space(R.riftkv_attention_pages_workspace_size(cache, 1, 2, top)), status)
    kk, vv = (x[:, 0].flatten(0, 1)[:int(lens), None].double().cpu() for x in (k, v))
    check(out[0], *attend(q[0].double().cpu(), kk, vv, 64 ** -0.5), q.dtype)
    assert int(status) == 0
