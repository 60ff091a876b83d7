"""Attention after a shared prefix and over listed pages against plain float64 forms."""
import math

import pytest
import torch

from tests.kv_ranges_testlib import TYPES, attend, attend_lists, check, filled, half_step, randn

pytestmark = pytest.mark.gpu

FORMS = [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"), ("f32", "bf16"), ("f32", "fp8"), ("f32", "int8")]


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def workspace(size):
    """As large as asked, and every byte of it NaN's."""
    return torch.full((max(size, 256),), 255, dtype=torch.uint8, device="cuda")


# ----------------------------------------------------------------------------- a shared prefix
def shared(R, P, q, prefix_len, lens, out=None, scale=None, stream=None, ws=None):
    """Sequence 0 of the pages is the prefix, the others are the callers'."""
    n, heads, _ = q.shape
    table = P.table[1:].contiguous()
    front = P.table[0, :-(-prefix_len // P.page)].contiguous()
    out = torch.full_like(q, 7.0) if out is None else out
    if ws is None:
        ws = workspace(R.riftkv_attention_shared_workspace_size(P.cache, n, heads, prefix_len, table.shape[1]))
    R.riftkv_attention_shared(P.cache, q, front, prefix_len, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, ws, P.status,
                              scale=scale, stream=stream)
    return out


def check_shared(P, q, prefix_len, lens, out, scale=None):
    """Of bf16 queries the prefix' weights are short by up to 2^-17: of each of their values' magnitudes."""
    kp, vp = P.rows(0, prefix_len)
    for i, n in enumerate(lens):
        k, v = P.rows(1 + i, n)
        keys, values, qd = torch.cat((kp, k)), torch.cat((vp, v)), q[i].double().cpu()
        scaled = q.shape[2] ** -0.5 if scale is None else scale
        o, e = attend(qd, keys, values, scaled)
        if q.dtype == torch.bfloat16:
            e = e + 2.0 ** -17 * attend(qd, keys, values.abs(), scaled)[0]
        check(out[i], o, e, q.dtype, f"sequence {i}")


@pytest.mark.parametrize("dt, store", FORMS)
@pytest.mark.parametrize("n_kv, group, hd, page, prefix, lens", [
    (2, 1, 128, 16, 35, [1, 0, 40, 33]),
    (1, 4, 64, 32, 100, [0]),
    (2, 3, 64, 16, 257, [5, 64, 1, 0, 31, 32, 17]),
    (1, 20, 128, 64, 130, [70, 3]),
    (2, 4, 128, 16, 1, [300, 2, 1]),
])
def test_shared(R, dt, store, n_kv, group, hd, page, prefix, lens):
    P = filled(R, store, n_kv, hd, page, [prefix] + lens, seed=page + hd, dtype=TYPES[dt] if store != "bf16" else torch.bfloat16)
    q = randn(5, len(lens), n_kv * group, hd, dtype=TYPES[dt], scale=2)
    out = shared(R, P, q, prefix, lens)
    check_shared(P, q, prefix, lens, out)
    assert int(P.status) == 0


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "f32"), ("f32", "int8")])
@pytest.mark.parametrize("n_kv, group, hd, page, prefix, seqs", [
    (1, 4, 128, 16, 700, 5), (2, 8, 64, 64, 1500, 9), (1, 5, 128, 32, 513, 13), (3, 1, 128, 16, 200, 40), (1, 1, 64, 16, 4100, 130),
    (1, 16, 128, 128, 2049, 17)])
def test_shared_many_rows(R, dt, store, n_kv, group, hd, page, prefix, seqs):
    """More query rows a key head than a tile has, and numbers of them that fill none."""
    lens = [(7 * i) % 50 for i in range(seqs)]
    P = filled(R, store, n_kv, hd, page, [prefix] + lens, seed=seqs)
    q = randn(6, seqs, n_kv * group, hd, dtype=TYPES[dt], scale=2)
    out = shared(R, P, q, prefix, lens)
    check_shared(P, q, prefix, lens, out)
    assert int(P.status) == 0


def test_shared_without_a_prefix_or_own_tokens(R):
    P = filled(R, "bf16", 2, 128, 16, [50, 20, 0, 3])
    q = randn(1, 3, 4, 128)
    out = shared(R, P, q, 0, [20, 0, 3])
    check_shared(P, q, 0, [20, 0, 3], out)
    assert bool((out[1] == 0).all())
    out = shared(R, P, q, 50, [0, 0, 0])
    check_shared(P, q, 50, [0, 0, 0], out)
    out = torch.full_like(q, 7.0)   # a table without columns
    none = torch.empty(3, 0, dtype=torch.int32, device="cuda")
    ws = workspace(R.riftkv_attention_shared_workspace_size(P.cache, 3, 4, 0, 0))
    R.riftkv_attention_shared(P.cache, q, P.table[0, :0], 0, none, torch.zeros(3, dtype=torch.int32, device="cuda"), out, ws, P.status)
    assert bool((out == 0).all()) and int(P.status) == 0


@pytest.mark.parametrize("store, prefix, longest", [("bf16", 40000, 300), ("int8", 20001, 9000), ("bf16", 100, 30000)])
def test_shared_long(R, store, prefix, longest):
    """Tokens that are split over many workgroups, among few and among many."""
    lens = [longest, 0, longest // 3]
    P = filled(R, store, 2, 128, 64, [prefix] + lens, seed=3)
    q = randn(8, 3, 8, 128, scale=3)
    out = shared(R, P, q, prefix, lens)
    check_shared(P, q, prefix, lens, out)
    again = shared(R, P, q, prefix, lens)
    assert torch.equal(out, again)


def test_shared_large_scores(R):
    """Scores up to some thousands, of either sign, and a scale of either sign or none."""
    P = filled(R, "bf16", 1, 128, 16, [90, 40, 0], spread=30.0)
    q = randn(9, 2, 4, 128, scale=10)
    for scale in (None, 1.0, -0.5, 0.0):
        out = shared(R, P, q, 90, [40, 0], scale=scale)
        check_shared(P, q, 90, [40, 0], out, scale=scale)


def test_shared_is_the_attention_over_one_table(R):
    """The same tokens as one context whose pages begin with the prefix': as riftkv_attention has it, to its own error."""
    page, prefix, lens = 32, 320, [50, 1, 333]
    P = filled(R, "bf16", 2, 128, page, [prefix] + lens, seed=4)
    q = randn(2, 3, 8, 128, scale=2)
    out = shared(R, P, q, prefix, lens)
    table = torch.cat((P.table[:1, :prefix // page].expand(3, -1), P.table[1:]), 1).contiguous()
    n = torch.tensor([prefix + x for x in lens], dtype=torch.int32, device="cuda")
    dense = torch.empty_like(q)
    ws = workspace(R.riftkv_attention_workspace_size(P.cache, 3, 8, table.shape[1]))
    R.riftkv_attention(P.cache, q, table, n, dense, ws, P.status)
    for i in range(3):
        k, v = P.rows(0, prefix), P.rows(1 + i, lens[i])
        o, e = attend(q[i].double().cpu(), torch.cat((k[0], v[0])), torch.cat((k[1], v[1])), 128 ** -0.5)
        off = (out[i].double() - dense[i].double()).abs().cpu()
        assert bool((off <= 2 * (e + half_step(torch.bfloat16) * o.abs() * 1.001)).all())


def test_shared_bad_pages_and_lengths(R):
    """On the device: the status, and NaN where it belongs."""
    P = filled(R, "bf16", 2, 128, 16, [100, 20, 40, 5])
    q = randn(1, 3, 4, 128)
    lens = [20, 40, 5]
    good = shared(R, P, q, 100, lens)
    table = P.table.clone()
    for bad in (-1, P.k.shape[0], 2 ** 31 - 1):
        P.table = table.clone()
        P.table[2, 1] = bad
        out = shared(R, P, q, 100, lens)
        assert int(P.status) == 2
        P.status.zero_()
        assert bool(torch.isnan(out[1]).all()) and torch.equal(out[::2], good[::2])
        P.table = table.clone()
        P.table[0, 6] = bad             # of the prefix
        out = shared(R, P, q, 100, lens)
        assert int(P.status) == 2 and bool(torch.isnan(out).all())
        P.status.zero_()
    P.table = table
    for n in (-1, P.table.shape[1] * 16 + 1, -2 ** 31, 2 ** 31 - 1):
        out = shared(R, P, q, 100, [20, n, 5])
        assert int(P.status) == 2
        P.status.zero_()
        assert bool(torch.isnan(out[1]).all()) and torch.equal(out[::2], good[::2])


# ----------------------------------------------------------------------------- listed pages
def listed(R, P, q, lens, lists, out=None, scale=None, stream=None, ws=None):
    n, heads, _ = q.shape
    out = torch.full_like(q, 7.0) if out is None else out
    if ws is None:
        ws = workspace(R.riftkv_attention_pages_workspace_size(P.cache, n, heads, lists.shape[2]))
    R.riftkv_attention_pages(P.cache, q, P.table, torch.tensor(lens, dtype=torch.int32, device="cuda"), lists.cuda(), out, ws, P.status,
                             scale=scale, stream=stream)
    return out


def random_lists(seed, lens, n_kv, top, page, order=True):
    """Some pages of every sequence for every key head, -1 behind them."""
    g = torch.Generator().manual_seed(seed)
    lists = torch.full((len(lens), n_kv, top), -1, dtype=torch.int32)
    for i, n in enumerate(lens):
        held = -(-n // page)
        for h in range(n_kv):
            pick = torch.randperm(held, generator=g)[:top]
            pick = pick.sort().values if order else pick
            lists[i, h, :len(pick)] = pick.int()
    return lists


@pytest.mark.parametrize("dt, store", FORMS)
@pytest.mark.parametrize("n_kv, group, hd, page, top, lens", [
    (2, 4, 128, 32, 4, [300, 1, 0, 65, 128]),
    (1, 1, 64, 16, 3, [47, 16, 33]),
    (3, 3, 64, 16, 7, [400, 90]),
    (1, 20, 128, 64, 2, [130, 500]),
    (4, 8, 128, 16, 1, [15, 200]),
])
def test_pages(R, dt, store, n_kv, group, hd, page, top, lens):
    P = filled(R, store, n_kv, hd, page, lens, seed=page + hd, dtype=TYPES[dt] if store != "bf16" else torch.bfloat16)
    q = randn(5, len(lens), n_kv * group, hd, dtype=TYPES[dt], scale=2)
    lists = random_lists(top, lens, n_kv, top, page)
    out = listed(R, P, q, lens, lists)
    check(out, *attend_lists(P, q, lens, lists), q.dtype)
    assert int(P.status) == 0


def test_pages_in_any_order(R):
    """Unsorted lists, gaps in them, places past the sequence's end, one that is listed twice."""
    lens, page = [210, 33, 16], 16
    P = filled(R, "bf16", 2, 128, page, lens)
    q = randn(4, 3, 4, 128, scale=2)
    lists = torch.tensor([[[13, 2, -1, 7, 0], [-5, -1, 13, 13, -2 ** 31]],
                          [[2, 1, 0, -1, 1], [-1, -1, -1, -1, -1]],
                          [[0, 5, 9, -1, 1], [3, 2, 1, -1, 13]]], dtype=torch.int32)
    out = listed(R, P, q, lens, lists)
    check(out, *attend_lists(P, q, lens, lists), q.dtype)
    assert int(P.status) == 0
    assert bool((out[1, 2:] == 0).all()) and bool((out[2, 2:] == 0).all())


@pytest.mark.parametrize("store, seqs, page, top, longest", [("bf16", 1, 32, 300, 20000), ("fp8", 3, 16, 513, 9000), ("bf16", 40, 64, 8, 3000),
                                                             ("int8", 2, 4096, 2, 9000), ("f32", 5, 128, 9, 2500)])
def test_pages_long(R, store, seqs, page, top, longest):
    """Lists that are split over workgroups, and not."""
    lens = [longest - 37 * i for i in range(seqs)]
    P = filled(R, store, 2, 128, page, lens, seed=top)
    q = randn(3, seqs, 8, 128, scale=2, dtype=torch.float32 if store == "f32" else torch.bfloat16)
    lists = random_lists(1, lens, 2, top, page)
    out = listed(R, P, q, lens, lists)
    check(out, *attend_lists(P, q, lens, lists), q.dtype)
    assert torch.equal(out, listed(R, P, q, lens, lists)) and int(P.status) == 0


def test_all_pages_is_the_dense_attention(R):
    lens, page = [500, 77, 0, 32], 32
    P = filled(R, "fp8", 2, 128, page, lens)
    q = randn(3, 4, 8, 128, scale=2)
    lists = random_lists(1, lens, 2, 16, page)
    out = listed(R, P, q, lens, lists)
    check(out, *attend_lists(P, q, lens, lists), q.dtype)
    dense = torch.empty_like(q)
    ws = workspace(R.riftkv_attention_workspace_size(P.cache, 4, 8, P.table.shape[1]))
    R.riftkv_attention(P.cache, q, P.table, torch.tensor(lens, dtype=torch.int32, device="cuda"), dense, ws, P.status)
    _, e = attend_lists(P, q, lens, lists)
    off = (out.double() - dense.double()).abs().cpu()
    assert bool((off <= 2 * (e + half_step(torch.bfloat16) * dense.double().abs().cpu() * 1.01)).all())


def test_pages_bad_places_and_lengths(R):
    lens, page = [100, 40, 64], 16
    P = filled(R, "bf16", 2, 128, page, lens)
    q = randn(4, 3, 4, 128)
    lists = random_lists(1, lens, 2, 3, page)
    good = listed(R, P, q, lens, lists)
    table = P.table.clone()
    for bad in (P.table.shape[1], 2 ** 31 - 1):
        x = lists.clone()
        x[1, 1, 0] = bad
        out = listed(R, P, q, lens, x)
        assert int(P.status) == 2
        P.status.zero_()
        assert bool(torch.isnan(out[1, 2:]).all()) and torch.equal(out[1, :2], good[1, :2]) and torch.equal(out[::2], good[::2])
    for bad in (-1, P.k.shape[0]):
        P.table = table.clone()
        P.table[1, int(lists[1, 0, 1])] = bad
        out = listed(R, P, q, lens, lists)
        assert int(P.status) == 2
        P.status.zero_()
        assert bool(torch.isnan(out[1, :2]).all()) and torch.equal(out[::2], good[::2])
    P.table = table
    for n in (-1, P.table.shape[1] * page + 1, 2 ** 31 - 1, -2 ** 31):
        out = listed(R, P, q, [100, n, 64], lists)
        assert int(P.status) == 2
        P.status.zero_()
        assert bool(torch.isnan(out[1]).all()) and torch.equal(out[::2], good[::2])


# ----------------------------------------------------------------------------- both
def both(R, P, q, lens, lists):
    """Either attention of the sequences, for the first one the others' prefix."""
    yield lambda out: shared(R, P, q[1:], lens[0], lens[1:], out=out[1:])
    yield lambda out: listed(R, P, q, lens, lists, out=out)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_strided_rows(R, dt):
    """Queries and outputs as slices of wider rows; nothing beside them changes."""
    lens = [90, 40, 5, 0]
    P = filled(R, "bf16", 2, 64, 16, lens)
    wide = randn(3, 4, 6 * 64, dtype=TYPES[dt])
    q = wide[:, 64:5 * 64].view(4, 4, 64)
    lists = random_lists(2, lens, 2, 3, 16)
    for call in both(R, P, q, lens, lists):
        room = torch.full((4, 8 * 64), 5.0, dtype=TYPES[dt], device="cuda")
        call(room[:, 128:384].view(4, 4, 64))
        tight = torch.full((4, 4, 64), 5.0, dtype=TYPES[dt], device="cuda")
        call(tight)
        assert torch.equal(room[:, 128:384].view(4, 4, 64), tight)
        assert bool((room[:, :128] == 5).all()) and bool((room[:, 384:] == 5).all())


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_numbers(R, value):
    """Among the tokens they reach their own heads' outputs, as a softmax has them; behind the last token, nothing."""
    lens, page = [60, 20, 33], 16
    P = filled(R, "bf16", 2, 128, page, lens)
    q = randn(4, 3, 4, 128)
    lists = torch.tensor([[[0, 1, 3]] * 2, [[0, 1, -1]] * 2, [[0, 2, -1]] * 2], dtype=torch.int32)
    clean = [torch.full_like(q, 7.0) for _ in range(2)]
    for out, call in zip(clean, both(R, P, q, lens, lists)):
        call(out)
    for x in (P.k, P.v):   # all that no token fills
        for i, n in enumerate(lens):
            last = int(P.table[i, n // page])
            x[last, :, n % page:] = value
    for out, call in zip(clean, both(R, P, q, lens, lists)):
        again = torch.full_like(q, 7.0)
        call(again)
        assert torch.equal(out, again)
    P.v[int(P.table[1, 0]), 1, 3, 5] = value                # a value of sequence 1, key head 1
    for out, call in zip(clean, both(R, P, q, lens, lists)):
        again = torch.full_like(q, 7.0)
        call(again)
        hit = ~torch.isfinite(again.float())
        want = torch.zeros_like(hit)
        want[1, 2:, 5] = True
        assert torch.equal(hit, want)
        assert torch.equal(again[~want], out[~want])
    P.k[int(P.table[1, 0]), 0, 3, 5] = value                # a key of key head 0: its outputs are NaN, or without that token
    for out, call, prefix in zip(clean, both(R, P, q, lens, lists), (lens[0], 0)):
        again = torch.full_like(q, 7.0)
        call(again)
        k = torch.cat((P.rows(0, prefix)[0], P.rows(1, lens[1])[0]))
        s = (q[1, :2].double().cpu() @ k[:, 0].t()) * 128 ** -0.5
        nan = torch.isnan(torch.softmax(s, -1)).any(-1)
        for j in range(2):
            assert bool(torch.isnan(again[1, j]).all()) == bool(nan[j])
        assert torch.equal(again[0], out[0]) and torch.equal(again[2], out[2])


@pytest.mark.parametrize("store", ["fp8", "int8"])
@pytest.mark.parametrize("prefix, seqs, group", [(60, 3, 2), (700, 3, 2), (700, 40, 2)])
def test_rows_of_8_bits_that_hold_nan(R, store, prefix, seqs, group):
    """Written as NaN: a key's makes its key head's outputs NaN, a value's too; the other key head keeps its bits."""
    lens = [(5 * i) % 30 for i in range(seqs)]
    P = filled(R, store, 2, 128, 16, [prefix] + lens, seed=9)
    q = randn(4, seqs, 2 * group, 128)
    good = shared(R, P, q, prefix, lens)
    check_shared(P, q, prefix, lens, good)
    lists = torch.arange(3, dtype=torch.int32).repeat(1, 2, 1)
    one = filled(R, store, 2, 128, 16, [40], seed=3)
    fine = listed(R, one, q[:1], [40], lists)
    for which in (0, 1):
        for pages, seq, n in ((P, 0, prefix), (one, 0, 40)):
            kv = randn(6, 1, 2, 2, 128)
            kv[0, which, 1, 77] = math.nan
            saved = [None if x is None else x.clone() for x in (pages.k.view(torch.uint8), pages.v.view(torch.uint8), pages.ks, pages.vs)]
            keep_k, keep_v = pages.rows(seq, n)
            kv[0, 0, 0], kv[0, 1, 0] = keep_k[n - 9, 0].cuda(), keep_v[n - 9, 0].cuda()      # key head 0 as it was
            pages.put(R, seq, kv[:, 0], kv[:, 1], first=n - 9)
            out = shared(R, P, q, prefix, lens) if pages is P else listed(R, one, q[:1], [40], lists)
            want = good if pages is P else fine
            assert bool(torch.isnan(out[:, group:]).all()) and torch.equal(out[:, :group], want[:, :group])
            for x, y in zip((pages.k.view(torch.uint8), pages.v.view(torch.uint8), pages.ks, pages.vs), saved):
                x.copy_(y)


def test_keys_of_minus_infinity(R):
    """Scores of -infinity alone: NaN, as a softmax gives; among others: weights of zero."""
    P = filled(R, "bf16", 1, 64, 16, [20, 20])
    q = torch.ones(2, 1, 64, dtype=torch.bfloat16, device="cuda")
    P.k[int(P.table[1, 0]), :, :, 0] = -math.inf
    P.k[int(P.table[1, 1]), :, :4, 0] = -math.inf
    lists = torch.tensor([[[0, 1]], [[0, 1]]], dtype=torch.int32)
    out = listed(R, P, q, [20, 20], lists)
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isfinite(out[0].float()).all())
    out = shared(R, P, q[1:], 20, [20])                      # after a prefix whose scores are numbers
    o, e = attend(q[1].double().cpu(), *P.rows(0, 20), 64 ** -0.5)
    check(out[0], o, e, q.dtype)


def test_other_streams_and_graphs(R):
    """On a stream of its own, and captured: every replay gives the eager call's bits, with inputs that change between them."""
    lens = [3000, 400, 77, 1]
    P = filled(R, "bf16", 2, 128, 32, lens, seed=1)
    q = randn(4, 4, 8, 128, scale=2)
    lists = random_lists(2, lens, 2, 12, 32)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    lists_d, table, front = lists.cuda(), P.table[1:].contiguous(), P.table[0, :-(-3000 // 32)].contiguous()
    wss = workspace(R.riftkv_attention_shared_workspace_size(P.cache, 3, 8, 3000, table.shape[1]))
    wsl = workspace(R.riftkv_attention_pages_workspace_size(P.cache, 4, 8, 12))
    a, b = torch.empty_like(q[1:]), torch.empty_like(q)

    def calls():
        R.riftkv_attention_shared(P.cache, q[1:], front, 3000, table, n[1:], a, wss, P.status)
        R.riftkv_attention_pages(P.cache, q, P.table, n, lists_d, b, wsl, P.status)

    calls()
    want = a.clone(), b.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.zero_(), b.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(3):
        q.copy_(randn(20 + i, 4, 8, 128, scale=2))
        n.copy_(torch.tensor([3000, 400 - 100 * i, 77, i], dtype=torch.int32))
        calls()
        want = a.clone(), b.clone()
        torch.cuda.synchronize()
        a.zero_(), b.zero_()
        wss.fill_(255), wsl.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((a, b), want):   # (the last sequence's second token is a row that was never written: NaN)
            assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    assert int(P.status) == 0


def test_two_streams_at_once(R):
    """Calls with a workspace each."""
    lens = [5000, 900, 33]
    P = filled(R, "int8", 2, 128, 64, lens, seed=1)
    qs = [randn(30 + i, 3, 8, 128, scale=2) for i in range(2)]
    lists = random_lists(2, lens, 2, 9, 64)
    want = [(shared(R, P, q[1:], 5000, lens[1:]), listed(R, P, q, lens, lists)) for q in qs]
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream() for _ in range(2)]
    lists_d, n = lists.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    table, front = P.table[1:].contiguous(), P.table[0].contiguous()
    buffers = [(workspace(R.riftkv_attention_shared_workspace_size(P.cache, 2, 8, 5000, table.shape[1])),
                workspace(R.riftkv_attention_pages_workspace_size(P.cache, 3, 8, 9)), torch.empty_like(q[1:]), torch.empty_like(q)) for q in qs]
    torch.cuda.synchronize()
    for _ in range(5):
        for q, s, (w1, w2, a, b) in zip(qs, streams, buffers):
            R.riftkv_attention_shared(P.cache, q[1:], front, 5000, table, n[1:], a, w1, P.status, stream=s)
            R.riftkv_attention_pages(P.cache, q, P.table, n, lists_d, b, w2, P.status, stream=s)
    torch.cuda.synchronize()
    for (a, b), (_, _, x, y) in zip(want, buffers):
        assert torch.equal(a, x) and torch.equal(b, y)
