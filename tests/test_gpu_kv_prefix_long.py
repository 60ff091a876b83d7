"""Long shared prefixes gone through for 128 query rows at a time: parts of more pages than a wave's registers hold the numbers of,
pages past 2^32 bytes, and 8-bit pages, which take this way from 900,000 (16 rows, token) pairs on."""
import math

import pytest
import torch

from tests.kv_ranges_testlib import TYPES, attend, check, filled, randn
from tests.test_gpu_kv_prefix_rows import check_prefix, held, pairs
from tests.test_gpu_kv_ranges import shared, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    yield R
    torch.cuda.empty_cache()


def enough(store):
    return 56000 if store == "bf16" else 900000


def parts(n_kv, group, hd, store, prefix, seqs):
    """First tile of 64 tokens of each part of the prefix, and the end."""
    wgs, tiles = n_kv * -(-seqs * group // 128), -(-prefix // 64)
    n = max(1, min((256 if store == "bf16" and hd == 128 else 384) // wgs, tiles // 2, 64))
    return [tiles * i // n for i in range(n + 1)]


WINDOWS = [("bf16", "bf16", 128, 16, 20000), ("bf16", "bf16", 64, 16, 19997), ("f32", "bf16", 128, 16, 20011), ("bf16", "bf16", 128, 32, 40000),
           ("bf16", "fp8", 128, 16, 19999), ("bf16", "int8", 128, 16, 20000), ("bf16", "int8", 64, 32, 40017)]


@pytest.mark.parametrize("dt, store, hd, page, prefix", WINDOWS)
def test_parts_of_many_pages(R, dt, store, hd, page, prefix):
    """Shuffled pages, more than 64 a part: their numbers are looked up anew on the way."""
    seqs, group = 64, 64
    at = parts(1, group, hd, store, prefix, seqs)
    assert pairs(1, group, prefix, seqs) > enough(store) and min(b - a for a, b in zip(at, at[1:])) * 64 > 80 * page
    lens = [i % 3 for i in range(seqs)]
    P = filled(R, store, 1, hd, page, [prefix] + lens, seed=page)
    q = randn(6, seqs, group, hd, dtype=TYPES[dt], scale=2)
    out = shared(R, P, q, prefix, lens)
    check_prefix(P, q, prefix, lens, out)
    assert torch.equal(out, shared(R, P, q, prefix, lens)) and int(P.status) == 0


@pytest.mark.parametrize("dt, store, hd, page, prefix", WINDOWS[:2] + WINDOWS[4:])
def test_bad_pages_of_long_parts(R, dt, store, hd, page, prefix):
    """Before, at and behind the 64th and the 128th page of a part."""
    seqs, group = 64, 64
    P = filled(R, store, 1, hd, page, [prefix] + [1] * seqs)
    q = randn(1, seqs, group, hd, dtype=TYPES[dt])
    lens = [1] * seqs
    good = shared(R, P, q, prefix, lens)
    at = parts(1, group, hd, store, prefix, seqs)
    first, behind = at[1] * 64 // page, at[2] * 64 // page
    table = P.table.clone()
    for place in [first + i for i in (-1, 0, 1, 59, 60, 61, 62, 63, 64, 65, 127, 128, 129)] + [behind - 1, (prefix - 1) // page]:
        assert place <= (prefix - 1) // page
        P.table = table.clone()
        P.table[0, place] = (-1, P.k.shape[0], 2 ** 31 - 1)[place % 3]
        out = shared(R, P, q, prefix, lens)
        assert int(P.status) == 2 and bool(torch.isnan(out).all()), place
        P.status.zero_()
    P.table = table
    assert torch.equal(shared(R, P, q, prefix, lens), good) and int(P.status) == 0


@pytest.mark.parametrize("store, hd, page, n_pages", [("bf16", 128, 16, 1_250_000), ("int8", 128, 16, 1_250_000)])
def test_places_past_32_bits(R, store, hd, page, n_pages):
    """The last pages of 40 or 20 GB, gone through many times over."""
    kv, group, dtype = 8, 2, torch.bfloat16 if store == "bf16" else torch.int8
    k = torch.zeros(n_pages, kv, page, hd, device="cuda", dtype=dtype)
    assert k.numel() * k.element_size() > 1 << 34
    scale = None if store == "bf16" else torch.full((n_pages, kv, page), 255, device="cuda", dtype=torch.uint8)
    cache, status = R.riftkv_cache(k, k, scale, scale), torch.zeros(1, dtype=torch.int32, device="cuda")
    at = [n_pages - 1, 3, n_pages - 70, 700_000, n_pages - 2]
    index = torch.tensor(at, device="cuda")
    if store == "bf16":
        rows = randn(3, len(at), kv, page, hd)
        k[index] = rows
        rows = rows.double()
    else:
        rows = torch.randint(-127, 128, (len(at), kv, page, hd), generator=torch.Generator().manual_seed(3)).cuda()
        by = torch.randint(118, 122, (len(at), kv, page), generator=torch.Generator().manual_seed(4)).cuda()
        k[index], scale[index] = rows.to(torch.int8), by.to(torch.uint8)
        rows = rows.double() * torch.exp2(by.double() - 127)[..., None]
    seqs, times = (40, 20) if store == "bf16" else (200, 60)
    n = page * len(at) * times - 3
    assert pairs(kv, group, n, seqs) > enough(store)
    q = randn(5, seqs, group * kv, hd, scale=2)
    out = torch.empty_like(q)
    front = torch.tensor(at * times, device="cuda", dtype=torch.int32)
    R.riftkv_attention_shared(cache, q, front, n, torch.empty(seqs, 0, device="cuda", dtype=torch.int32),
                              torch.zeros(seqs, device="cuda", dtype=torch.int32), out,
                              workspace(R.riftkv_attention_shared_workspace_size(cache, seqs, group * kv, n, 0)), status)
    every = rows.transpose(1, 2).flatten(0, 1).repeat(times, 1, 1)[:n].cpu()
    for i in (0, 17, seqs - 1):
        check(out[i], *attend(q[i].double().cpu(), every, every, hd ** -0.5), q.dtype)
    assert int(status) == 0


# ----------------------------------------------------------------------------- 8-bit pages
SHAPES = [(1, 64, 128, 32, 9001, 26), (2, 50, 64, 16, 5125, 33), (1, 2048, 128, 128, 7050, 1), (5, 3, 64, 64, 4400, 220)]


@pytest.mark.parametrize("store", ["fp8", "int8"])
@pytest.mark.parametrize("shape", SHAPES)
def test_8_bit_pages(R, store, shape):
    n_kv, group, hd, page, prefix, seqs = shape
    assert pairs(n_kv, group, prefix, seqs) > enough(store)
    lens = [(7 * i) % 50 for i in range(seqs)]
    P = filled(R, store, n_kv, hd, page, [prefix] + lens, seed=seqs)
    q = randn(6, seqs, n_kv * group, hd, scale=2)
    out = shared(R, P, q, prefix, lens)
    check_prefix(P, q, prefix, lens, out)
    assert torch.equal(out, shared(R, P, q, prefix, lens)) and int(P.status) == 0


@pytest.mark.parametrize("store", ["fp8", "int8"])
@pytest.mark.parametrize("prefix", [3583, 3584, 3585, 3599, 3600, 3601, 3647, 3648, 3649])
def test_8_bit_ends_of_the_prefix(R, store, prefix):
    """Whole tiles, a token more or fewer, pages that end inside a tile and pieces of 16 tokens that none of them is in."""
    n_kv, seqs = 16, 32
    assert pairs(n_kv, 8, prefix, seqs) > enough(store)
    P = filled(R, store, n_kv, 64, 16, [prefix] + [1] * seqs, seed=prefix)
    q = randn(6, seqs, n_kv * 8, 64, scale=3)
    out = shared(R, P, q, prefix, [1] * seqs)
    check_prefix(P, q, prefix, [1] * seqs, out)


@pytest.mark.parametrize("store", ["fp8", "int8"])
@pytest.mark.parametrize("scale", [1.0, -0.5, 0.0])
def test_8_bit_large_scores(R, store, scale):
    prefix, seqs = 9001, 26
    P = filled(R, store, 1, 128, 16, [prefix] + [3] * seqs, spread=30.0)
    q = randn(9, seqs, 64, 128, scale=10)
    out = shared(R, P, q, prefix, [3] * seqs, scale=scale)
    check_prefix(P, q, prefix, [3] * seqs, out, scale=scale)


@pytest.mark.parametrize("store", ["fp8", "int8"])
@pytest.mark.parametrize("at", [0, 4500, 9000])
def test_8_bit_rows_that_hold_nan(R, store, at):
    """A key's or a value's NaN reaches all its key head's outputs, and no other key head's."""
    prefix, seqs, lens = 9001, 26, [3] * 26
    P = filled(R, store, 2, 64, 32, [prefix] + lens, seed=9)
    q = randn(4, seqs, 128, 64)
    good = shared(R, P, q, prefix, lens)
    k, v = (x[at].clone() for x in held(P, 0, prefix))
    for which in (0, 1):
        kv = torch.stack((k, v))[None].to(torch.bfloat16).cuda()
        kv[0, which, 1, 7] = math.nan
        P.put(R, 0, kv[:, 0], kv[:, 1], first=at)
        out = shared(R, P, q, prefix, lens)
        assert bool(torch.isnan(out[:, 64:]).all()) and torch.equal(out[:, :64], good[:, :64])
    assert int(P.status) == 0


@pytest.mark.parametrize("store", ["fp8", "int8"])
def test_8_bit_in_a_graph(R, store):
    prefix, seqs, lens = 9001, 26, [3] * 26
    P = filled(R, store, 1, 128, 16, [prefix] + lens)
    q, out = randn(1, seqs, 64, 128), torch.empty(seqs, 64, 128, dtype=torch.bfloat16, device="cuda")
    table, front = P.table[1:].contiguous(), P.table[0, :-(-prefix // 16)].contiguous()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = workspace(R.riftkv_attention_shared_workspace_size(P.cache, seqs, 64, prefix, table.shape[1]))

    def call():
        R.riftkv_attention_shared(P.cache, q, front, prefix, table, n, out, ws, P.status)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        q.copy_(randn(10 + i, seqs, 64, 128, scale=2))
        out.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, shared(R, P, q, prefix, lens))
        check_prefix(P, q, prefix, lens, out)
    assert int(P.status) == 0
