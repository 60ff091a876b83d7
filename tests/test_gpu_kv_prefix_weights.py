"""How exact the weights of a shared prefix are where it is gone through for 128 query rows at a time: as everywhere else."""
import math

import pytest
import torch

from tests.kv_ranges_testlib import TYPES, filled, half_step
from tests.test_gpu_kv_prefix_rows import check_prefix, held, pairs
from tests.test_gpu_kv_ranges import shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


# Sequences with 64 rows of one key head each: enough (16 rows, token) pairs for 128 rows at a time.
SEQS, GROUP, HD = 26, 64, 64
LENGTH = {"bf16": 4161, "fp8": 9000, "int8": 9000}


def terms(x):
    """Three bf16 numbers that add up to x, to 2^-24 of it."""
    out = []
    for _ in range(3):
        t = float(torch.tensor(x, dtype=torch.float64).bfloat16())
        out.append(t)
        x -= t
    return out


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "bf16")])
def test_every_bit_of_a_weight(R, dt, store):
    """A weight of 0.5 (1 + 2^-8 + 2^-16), halfway between two sums of two bf16 numbers and 2^-16 from either, against
    weights that two numbers hold: what is left of the sum is the last 2^-17."""
    prefix = LENGTH[store]
    assert pairs(1, GROUP, prefix, SEQS) > (56000 if store == "bf16" else 900000)
    P = filled(R, store, 1, HD, 16, [prefix] + [0] * SEQS)
    # scores by token: 0; the odd weight's; those of 0.5; all others none at all
    q = torch.zeros(SEQS, GROUP, HD, dtype=torch.float64)
    for i, x in enumerate(terms(math.log(0.5 * (1 + 2.0 ** -8 + 2.0 ** -16))) + terms(math.log(0.5)) + [-200.0]):
        q[:, :, i] = x
    q = q.to(TYPES[dt]).cuda()
    k = torch.zeros(prefix, 1, HD, dtype=torch.bfloat16)
    v = torch.zeros(prefix, 1, HD, dtype=torch.bfloat16)
    k[:, 0, 6] = 1
    place = (70, 77, 130, 131)                                  # one tile's two halves, and the next one
    k[place, 0] = 0
    k[place[1], 0, 0:3] = 1
    k[place[2:], 0, 3:6] = 1
    v[place[1]] = 1
    v[place[2]] = -1
    v[place[3]] = -2.0 ** -8
    P.put(R, 0, k.cuda(), v.cuda())
    out = shared(R, P, q, prefix, [0] * SEQS, scale=1.0)
    kd, vd = (x[:, 0].cpu() for x in held(P, 0, prefix))
    w = torch.softmax(kd @ q[0, 0].double().cpu(), 0)
    want = w @ vd
    # Scores of three products and two roundings, of up to 0.7; an exponential of 2^-22 and twice the scores' error; four
    # weights that are not zero are added up, in parts of the prefix and then the parts; two more roundings.
    err = (2 * (3 + 2) * 2.0 ** -24 * 0.7 + 2.0 ** -22 + 12 * 2.0 ** -24) * (w @ vd.abs()) + half_step(TYPES[dt]) * want.abs()
    off = (out.double().cpu() - want).abs()
    assert bool((off <= err).all()), float((off / err).max())
    assert float(err[0]) < 0.5 * 2.0 ** -17 * float(w[place[0]])      # a weight short by 2^-17 of it would be seen


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "bf16")])
@pytest.mark.parametrize("exponent", [-100, 114])
def test_large_and_small_values(R, dt, store, exponent):
    """Values of 2^114, whose sum over all tokens is below 2^128, as a running maximum's sum is: scores that are 2^7.8 apart in
    every tile, the smaller ones first.  And values that are as small."""
    prefix = LENGTH[store]
    assert pairs(1, GROUP, prefix, SEQS) > (56000 if store == "bf16" else 900000) and prefix * 1.125 * 2.0 ** 114 < 2.0 ** 128
    P = filled(R, store, 1, HD, 16, [prefix] + [0] * SEQS)
    k = torch.zeros(prefix, 1, HD)
    k[:, 0, 0] = (torch.arange(prefix) % 64 >= 32).float()
    v = 1 + torch.randint(0, 2, (prefix, 1, HD), generator=torch.Generator().manual_seed(3)) / 8
    v = torch.ldexp(v, torch.tensor(exponent))
    P.put(R, 0, k.bfloat16().cuda(), v.bfloat16().cuda())
    q = torch.zeros(SEQS, GROUP, HD, dtype=TYPES[dt], device="cuda")
    q[:, :, 0] = 7.8 * math.log(2)
    out = shared(R, P, q, prefix, [0] * SEQS, scale=1.0)
    assert bool(torch.isfinite(out).all())
    out = out.double() * 2.0 ** -exponent                        # (the check's smallest bound is 1e-30)
    P.v = (P.v.double() * 2.0 ** -exponent).to(P.store) if P.vs is None else P.v
    if P.vs is not None:
        P.vs = (P.vs.int() - exponent).to(torch.uint8)
    check_prefix(P, q, prefix, [0] * SEQS, out, scale=1.0)


def test_values_below_the_weights_bits(R):
    """8-bit rows whose scale is 2^-100: a weight of 2^-8 or more times it still has all its bits above 2^-133."""
    prefix = LENGTH["int8"]
    P = filled(R, "int8", 1, HD, 16, [prefix] + [0] * SEQS)
    k = torch.randn(prefix, 1, HD, generator=torch.Generator().manual_seed(5)).bfloat16()
    v = torch.ldexp(torch.randint(64, 128, (prefix, 1, HD), generator=torch.Generator().manual_seed(6)).float(), torch.tensor(-100))
    P.put(R, 0, k.cuda(), v.bfloat16().cuda())
    q = torch.randn(SEQS, GROUP, HD, generator=torch.Generator().manual_seed(7)).bfloat16().cuda()
    out = shared(R, P, q, prefix, [0] * SEQS)
    P.vs = (P.vs.int() + 100).to(torch.uint8)
    check_prefix(P, q, prefix, [0] * SEQS, out.double() * 2.0 ** 100)


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "bf16")])
@pytest.mark.parametrize("exponent", [10, 20, 34, 60])
@pytest.mark.parametrize("scale", [1.0, -0.3])
@pytest.mark.parametrize("seqs, prefix", [(SEQS, None), (2, 700), (2, 200)])
def test_scores_of_any_size(R, dt, store, exponent, scale, seqs, prefix):
    """Scores of 2^10 to 2^60, whose last bit is worth far more than an exponent can be: the tokens of the largest one share all
    the weight.  By 128 rows, by 16, and a prefix that every sequence walks."""
    prefix = prefix or LENGTH[store]
    P = filled(R, store, 1, HD, 16, [prefix] + [0] * seqs)
    g = torch.Generator().manual_seed(exponent)
    k = torch.zeros(prefix, 1, HD)
    k[:, 0, 0] = torch.randint(-100, 101, (prefix,), generator=g).float() / 64
    k[:, 0, 1] = 1
    P.put(R, 0, k.bfloat16().cuda(), torch.randn(prefix, 1, HD, generator=g).bfloat16().cuda())
    q = torch.zeros(seqs, GROUP, HD, dtype=TYPES[dt], device="cuda")
    q[:, ::2, 0], q[:, 1::2, 0] = 2.0 ** exponent, -1.25 * 2.0 ** exponent
    q[:, ::3, 1] = 1.0
    out = shared(R, P, q, prefix, [0] * seqs, scale=scale)
    kd, vd = (x[:, 0].cpu() for x in held(P, 0, prefix))
    for row in range(6):
        s = (kd @ q[0, row].double().cpu()) * scale
        assert exponent < 20 or float(s.max() - s[s < s.max()].max()) > 1000
        if exponent >= 20:
            best = s == s.max()
            want = vd[best].mean(0)
            err = (int(best.sum()) + 8) * 2.0 ** -24 * vd[best].abs().mean(0) + half_step(TYPES[dt]) * want.abs() * (1 + 1e-3)
            assert bool(((out[:, row].double().cpu() - want).abs() <= err).all()), row
    if exponent < 20:
        check_prefix(P, q, prefix, [0] * seqs, out, scale=scale)
