"""A shared prefix gone through for 128 query rows at a time, which calls with much to do take: against plain float64 forms, and where
it can go wrong."""
import math

import pytest
import torch

from tests.kv_ranges_testlib import TYPES, check, filled, randn
from tests.test_gpu_kv_ranges import shared, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def held(P, seq, n):
    """Pages.rows, gathered and widened on the GPU: k, v [n][n_kv][hd] in float64."""
    pages = P.table[seq, :-(-n // P.page)].long()
    out = []
    for x, s in ((P.k, P.ks), (P.v, P.vs)):
        y = x.view(torch.uint8)[pages].view(P.store).float().double()
        if s is not None:
            b = s[pages].double()
            y = y * torch.where(b == 255, torch.full_like(b, math.nan), torch.exp2(b - 127))[..., None]
        out.append(y.transpose(1, 2).flatten(0, 1)[:n])
    return out


def check_prefix(P, q, prefix, lens, out, scale=None):
    """Against float64, all sequences of a key head at once; the error of a float32 evaluation as `attend` has it, and of bf16 queries
    the 2^-17 of every weight of the prefix."""
    n, heads, hd = q.shape
    n_kv, wide = P.k.shape[1], max(lens)
    g, scale = heads // n_kv, hd ** -0.5 if scale is None else scale
    kp, vp = held(P, 0, prefix)
    own = torch.zeros(2, n, wide, n_kv, hd, dtype=torch.float64, device="cuda")
    for i, x in enumerate(lens):
        if x:
            own[0, i, :x], own[1, i, :x] = held(P, 1 + i, x)
    there = torch.arange(wide, device="cuda") < torch.tensor(lens, device="cuda")[:, None]
    for h in range(n_kv):
        qh = q[:, h * g:(h + 1) * g].double()

        def products(a):
            x, y = a(qh), [a(k[..., h, :]).transpose(-1, -2).contiguous() for k in (kp, own[0])]
            return torch.cat((x @ y[0], x @ y[1]), -1)

        mask = torch.cat((torch.ones(n, prefix, dtype=torch.bool, device="cuda"), there), 1)[:, None]
        w = torch.softmax((products(lambda x: x) * scale).masked_fill(~mask, -math.inf), -1)

        def sums(a):
            return w[..., :prefix] @ a(vp[:, h].contiguous()), w[..., prefix:] @ a(own[1][:, :, h].contiguous())

        front, tail = sums(torch.abs)
        e_score = (hd + 4) * 2.0 ** -24 * (products(torch.abs) * abs(scale)).masked_fill(~mask, 0).amax(-1)
        tokens = prefix + torch.tensor(lens, device="cuda")[:, None]
        e = (2 * e_score + 2.0 ** -21 + (tokens + 8) * 2.0 ** -24)[..., None] * (front + tail)
        if q.dtype == torch.bfloat16:
            e = e + 2.0 ** -17 * front
        check(out[:, h * g:(h + 1) * g], sum(sums(lambda x: x)).cpu(), e.cpu(), q.dtype, f"key head {h}")


def pairs(n_kv, group, prefix, seqs):
    """What the choice is made by: 16 rows of a key head, and a token."""
    return n_kv * -(-seqs * group // 16) * prefix


LARGE = [(1, 64, 128, 32, 4161, 26), (2, 50, 64, 16, 2053, 33), (1, 2048, 128, 128, 3400, 1), (5, 3, 64, 64, 2049, 220)]
SMALLER = [(1, 16, 128, 16, 4100, 15), (3, 1, 64, 256, 700, 500), (32, 1, 128, 32, 257, 130)]


@pytest.mark.parametrize("dt, store, shape", [(dt, store, s) for dt, store, shapes in (
    ("bf16", "bf16", SMALLER + LARGE[:2]), ("f32", "bf16", SMALLER[:2] + LARGE[1:3]), ("bf16", "fp8", LARGE), ("bf16", "int8", LARGE)) for s in shapes])
def test_prefix(R, dt, store, shape):
    n_kv, group, hd, page, prefix, seqs = shape
    assert pairs(n_kv, group, prefix, seqs) > (56000 if store == "bf16" else 400000)
    lens = [(7 * i) % 50 for i in range(seqs)]
    P = filled(R, store, n_kv, hd, page, [prefix] + lens, seed=seqs)
    q = randn(6, seqs, n_kv * group, hd, dtype=TYPES[dt], scale=2)
    out = shared(R, P, q, prefix, lens)
    check_prefix(P, q, prefix, lens, out)
    assert torch.equal(out, shared(R, P, q, prefix, lens)) and int(P.status) == 0


@pytest.mark.parametrize("store, rows", [("bf16", 32), ("int8", 256)])
@pytest.mark.parametrize("prefix", [2047, 2048, 2049, 2063, 2064, 2065, 2111, 2112, 2113])
def test_ends_of_the_prefix(R, store, rows, prefix):
    """Whole tiles, a token more or fewer, pages that end inside a tile and pieces of 16 tokens that none of them is in."""
    n_kv = 16
    assert pairs(n_kv, 8, prefix, rows // 8) > (56000 if store == "bf16" else 400000)
    P = filled(R, store, n_kv, 64, 16, [prefix] + [1] * (rows // 8), seed=prefix)
    q = randn(6, rows // 8, n_kv * 8, 64, scale=3)
    out = shared(R, P, q, prefix, [1] * (rows // 8))
    check_prefix(P, q, prefix, [1] * (rows // 8), out)


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "int8")])
@pytest.mark.parametrize("scale", [1.0, -0.5, 0.0])
def test_large_scores(R, dt, store, scale):
    """Scores up to some thousands, of either sign, and a scale of either sign or none."""
    prefix, seqs = 4161, 26
    P = filled(R, store, 1, 128, 16, [prefix] + [3] * seqs, spread=30.0)
    q = randn(9, seqs, 64, 128, dtype=TYPES[dt], scale=10)
    out = shared(R, P, q, prefix, [3] * seqs, scale=scale)
    check_prefix(P, q, prefix, [3] * seqs, out, scale=scale)


@pytest.mark.parametrize("store", ["bf16", "int8"])
def test_rising_scores(R, store):
    """Every tile's scores above all before it: sums are rescaled each time."""
    prefix, seqs, hd = 4161, 26, 64
    P = filled(R, store, 1, hd, 16, [prefix] + [0] * seqs)
    k = torch.zeros(prefix, 1, hd, dtype=torch.bfloat16)
    k[:, 0, 0] = torch.arange(prefix) / 8
    k[:, 0, 1:] = torch.randn(prefix, hd - 1, generator=torch.Generator().manual_seed(1)) / 8
    v = torch.randn(prefix, 1, hd, generator=torch.Generator().manual_seed(2)).bfloat16()
    P.put(R, 0, k.cuda(), v.cuda())
    q = randn(3, seqs, 64, hd)
    q[:, ::2, 0] = 8.0
    q[:, 1::2, 0] = -8.0
    out = shared(R, P, q, prefix, [0] * seqs)
    check_prefix(P, q, prefix, [0] * seqs, out)


@pytest.mark.parametrize("store", ["bf16", "fp8", "int8"])
def test_bad_pages(R, store):
    """On the device: the status, and NaN for all; the table's entries behind the prefix are not read."""
    prefix, seqs = 4161, 26
    P = filled(R, store, 1, 128, 16, [prefix] + [3] * seqs)
    q = randn(1, seqs, 64, 128)
    lens = [3] * seqs
    good = shared(R, P, q, prefix, lens)
    table = P.table.clone()
    for place in (0, 63, 64, 100, prefix // 16):
        for bad in (-1, P.k.shape[0], 2 ** 31 - 1):
            P.table = table.clone()
            P.table[0, place] = bad
            out = shared(R, P, q, prefix, lens)
            assert int(P.status) == 2 and bool(torch.isnan(out).all())
            P.status.zero_()
    P.table = table
    assert torch.equal(shared(R, P, q, prefix, lens), good) and int(P.status) == 0


@pytest.mark.parametrize("store", ["bf16", "int8"])
@pytest.mark.parametrize("at", [0, 2000, 4160])
def test_rows_that_hold_nan(R, store, at):
    """A key's or a value's NaN reaches all its key head's outputs (a value's in its own place), and no other key head's."""
    prefix, seqs, lens = 4161, 26, [3] * 26
    P = filled(R, store, 2, 64, 32, [prefix] + lens, seed=9)
    q = randn(4, seqs, 128, 64)
    good = shared(R, P, q, prefix, lens)
    k, v = (x[at].clone() for x in held(P, 0, prefix))
    for which in (0, 1):
        kv = torch.stack((k, v))[None].to(torch.bfloat16).cuda()    # [1][2][key heads][64]
        kv[0, which, 1, 7] = math.nan
        P.put(R, 0, kv[:, 0], kv[:, 1], first=at)
        out = shared(R, P, q, prefix, lens)
        hit = out[:, 64:] if which == 0 or store == "int8" else out[:, 64:, 7]
        assert bool(torch.isnan(hit).all()) and torch.equal(out[:, :64], good[:, :64])
        if which == 1 and store == "bf16":
            assert int(torch.isnan(out).sum()) == out.shape[0] * 64
    assert int(P.status) == 0


def test_scores_of_minus_infinity(R):
    """In a whole part of the prefix: no weight; in all of it and without other tokens: NaN, as a softmax has it."""
    prefix, seqs, hd = 4161, 26, 64
    P = filled(R, "bf16", 1, hd, 16, [prefix] + [0] * (seqs - 1) + [5])
    q = randn(3, seqs, 64, hd)
    q[:, :, 0] = 1.0
    k, v = held(P, 0, prefix)
    for n in (100, 3000, prefix):
        k2 = k.clone()
        k2[:n, 0, 0] = -math.inf
        P.put(R, 0, k2.bfloat16().cuda(), v.bfloat16().cuda())
        out = shared(R, P, q, prefix, [0] * (seqs - 1) + [5])
        if n < prefix:
            check_prefix(P, q, prefix, [0] * (seqs - 1) + [5], out)
        else:
            assert bool(torch.isnan(out[:-1]).all()) and bool(torch.isfinite(out[-1].float()).all())


@pytest.mark.parametrize("store", ["bf16", "fp8"])
def test_in_a_graph(R, store):
    """Captured and replayed with other inputs in place, eager calls of other shapes between."""
    prefix, seqs, lens = 4161, 26, [3] * 26
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
    for i in range(4):
        q.copy_(randn(10 + i, seqs, 64, 128, scale=2))
        out.fill_(7.0)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, shared(R, P, q, prefix, lens))
        check_prefix(P, q, prefix, lens, out)
    assert int(P.status) == 0
