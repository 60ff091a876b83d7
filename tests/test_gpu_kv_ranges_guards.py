"""Workspaces of exactly the reported size with a pattern behind them, a prefix' workgroups before items that take several launches, and
bounds of large pages."""
import pytest
import torch

from tests.kv_ranges_testlib import TYPES, attend_lists, bounds_of, check, filled, half_step, randn
from tests.test_gpu_kv_select import i32, new_bounds, same

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    yield R
    torch.cuda.empty_cache()


class Guarded:
    """A workspace, and what nothing may change behind it."""

    def __init__(self, size):
        self.all = torch.full((size + GUARD,), 165, dtype=torch.uint8, device="cuda")
        self.space = self.all[:size]
        self.space.fill_(255)

    def kept(self):
        return bool((self.all[self.space.numel():] == 165).all())


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "int8"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n_kv, group, seqs", [(1, 17, 3), (2, 17, 70), (4, 1, 5), (8, 1, 130), (3, 33, 40), (1, 16, 1), (1, 64, 26)])
@pytest.mark.parametrize("prefix", [0, 100, 256, 257, 2049, 9001])
def test_shared_keeps_to_its_workspace(R, dt, store, n_kv, group, seqs, prefix):
    lens = [(37 * i) % 300 for i in range(seqs)]
    P = filled(R, store, n_kv, 64, 16, [max(prefix, 1)] + lens, seed=seqs)
    q = randn(2, seqs, n_kv * group, 64, dtype=TYPES[dt])
    table, front = P.table[1:].contiguous(), P.table[0, :-(-prefix // 16)].contiguous()
    ws = Guarded(R.riftkv_attention_shared_workspace_size(P.cache, seqs, n_kv * group, prefix, table.shape[1]))
    out = torch.full_like(q, 7.0)
    R.riftkv_attention_shared(P.cache, q, front, prefix, table, i32(lens), out, ws.space, P.status)
    assert ws.kept() and bool(torch.isfinite(out.float()).all()) and int(P.status) == 0


@pytest.mark.parametrize("dt, store", [("bf16", "fp8"), ("f32", "f32")])
@pytest.mark.parametrize("n_kv, group, seqs, top", [(1, 17, 3, 100), (8, 1, 16, 64), (8, 4, 16, 40), (2, 33, 1, 700), (4, 1, 64, 90), (1, 1, 1, 1)])
def test_lists_keep_to_their_workspace(R, dt, store, n_kv, group, seqs, top):
    lens = [1600 - 31 * (i % 40) for i in range(seqs)]
    P = filled(R, store, n_kv, 64, 16, lens, seed=top)
    q = randn(2, seqs, n_kv * group, 64, dtype=TYPES[dt])
    bounds, out = new_bounds(P), torch.full_like(q, 7.0)
    R.riftkv_page_bounds(P.cache, bounds, P.table, i32(lens), P.status)
    lists = torch.full((seqs, n_kv, top), -5, device="cuda", dtype=torch.int32)
    ws = Guarded(R.riftkv_select_pages_workspace_size(P.cache, seqs, P.table.shape[1]))
    R.riftkv_select_pages(P.cache, bounds, q, P.table, i32(lens), lists, ws.space, P.status, keep_first=0)
    assert ws.kept()
    ws = Guarded(R.riftkv_attention_pages_workspace_size(P.cache, seqs, n_kv * group, top))
    R.riftkv_attention_pages(P.cache, q, P.table, i32(lens), lists, out, ws.space, P.status)
    assert ws.kept() and bool(torch.isfinite(out.float()).all()) and int(P.status) == 0


@pytest.mark.parametrize("n_kv, seqs", [(16, 4), (13, 5), (17, 10), (19, 9)])
@pytest.mark.parametrize("top", [23, 24, 39, 40])
def test_float32_lists_in_parts_and_whole(R, n_kv, seqs, top):
    """64, 65, 170 and 171 lists of 12 and 20 tiles, and of one less."""
    lens = [16 * top + 40 - i for i in range(seqs)]
    P = filled(R, "f32", n_kv, 64, 16, lens, seed=top)
    q = randn(2, seqs, n_kv, 64, dtype=torch.float32, scale=2)
    g = torch.Generator().manual_seed(seqs)
    lists = torch.stack([torch.stack([torch.randperm(-(-n // 16), generator=g)[:top] for _ in range(n_kv)]) for n in lens]).int().cuda()
    out = torch.full_like(q, 7.0)
    ws = Guarded(R.riftkv_attention_pages_workspace_size(P.cache, seqs, n_kv, top))
    R.riftkv_attention_pages(P.cache, q, P.table, i32(lens), lists, out, ws.space, P.status)
    check(out, *attend_lists(P, q, lens, lists), q.dtype)
    assert ws.kept() and int(P.status) == 0


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("f32", "f32")])
def test_a_prefix_before_items_of_many_launches(R, dt, store):
    """33,553,920 (sequence, key head) pairs after 300 tokens, which go by 128 rows (bf16) or 16: equal weights of values that are
    the same in all of the prefix, and of one token more or none."""
    n, kv, hd, prefix, dtype = 65535, 512, 64, 300, TYPES[dt]
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(5, kv, 512, hd, device="cuda", dtype=dtype, generator=g)
    v = torch.randn(5, kv, 512, hd, device="cuda", dtype=dtype, generator=g)
    v[4] = v[4, :, :1]
    cache, status = R.riftkv_cache(k, v), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(n, kv, hd, device="cuda", dtype=dtype)
    a = torch.arange(n, device="cuda", dtype=torch.int32)
    table, lens = (a % 4)[:, None].contiguous(), (a % 3 != 0).int().contiguous()
    out = torch.full_like(q, 7.0)
    size = R.riftkv_attention_shared_workspace_size(cache, n, kv, prefix, 1)
    ws = Guarded(size)
    R.riftkv_attention_shared(cache, q, i32([4]), prefix, table, lens, out, ws.space, status)
    assert ws.kept() and int(status) == 0
    front = v[4, :, 0].double()
    for page in range(4):
        for held in (0, 1):
            want = (prefix * front + held * v[page, :, 0].double()) / (prefix + held)
            # the sums of 301 equal weights in float32, and the output's rounding
            bound = (prefix + 8) * 2.0 ** -24 * (prefix * front.abs() + held * v[page, :, 0].double().abs()) / (prefix + held)
            bound = bound + half_step(dtype) * want.abs() * (1 + 1e-3)
            at = ((a % 4 == page) & (lens == held)).nonzero()[:, 0]
            for piece in at.split(1024):
                assert bool(((out[piece].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("store", ["bf16", "f32", "fp8", "int8"])
@pytest.mark.parametrize("hd, page, lens, begins", [
    (128, 512, [1024, 511, 513], None),
    (64, 1024, [1, 1023, 2500], [0, 1022, 2100]),
    (128, 4096, [4096, 5001], [4095, 5000]),
    (64, 4096, [4095, 8193], [17, 4096]),
])
def test_bounds_of_large_pages(R, store, hd, page, lens, begins):
    P = filled(R, store, 2, hd, page, lens, seed=hd)
    b = new_bounds(P)
    want = b.clone()
    for i, n in enumerate(lens):
        first = 0 if begins is None else begins[i]
        for p in range(first // page, -(-n // page)):
            want[int(P.table[i, p])] = bounds_of(P, i, n, p).to(b.dtype).cuda()
    R.riftkv_page_bounds(P.cache, b, P.table, i32(lens), P.status, begins=None if begins is None else i32(begins))
    assert same(b, want) and int(P.status) == 0
