"""The same sequences under tables of other widths: other kernels, the same values to the float32 bound, and the same bits
wherever width and lengths are the same."""
import pytest
import torch

from tests.test_gpu_kv import TYPES, attention, check, filled, randn
from tests.test_gpu_kv_decode import GATE, SMALL, Run
from tests.rift_testlib import rowwise_rel_err

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    R.load()
    return R


def widened(table, columns):
    wide = torch.full((table.shape[0], columns), 1 << 30, dtype=torch.int32, device="cuda")   # entries that are not read
    wide[:, :table.shape[1]] = table
    return wide


@pytest.mark.parametrize("dt, store", [("bf16", "bf16"), ("bf16", "fp8"), ("f32", "int8"), ("f32", "f32")])
@pytest.mark.parametrize("hd, n_kv, group, lens", [(128, 2, 4, [64, 17, 0, 50]), (64, 3, 1, [60, 1]), (128, 1, 18, [33, 64, 64])])
def test_attention_under_wider_tables(R, dt, store, hd, n_kv, group, lens):
    P = filled(R, store, n_kv, hd, 16, lens, seed=41, dtype=TYPES[dt])
    q = randn(14, len(lens), n_kv * group, hd, dtype=TYPES[dt], scale=2)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for columns in (4, 8, 16, 24, 32, 33, 64, 65, 5000):     # 64 tokens to 80,000
        table = widened(P.table, columns)
        out, again = attention(R, P, q, n, table=table), attention(R, P, q, n, table=table)
        torch.cuda.synchronize()
        assert int(P.status) == 0 and torch.equal(out, again), columns
        check(P, q, out, lens)


@pytest.mark.parametrize("pages_of", ["bf16", "int8"])
def test_a_step_under_wider_tables(R, pages_of):
    r = Run(R, SMALL, 2, [40, 3, 21], pages_of)
    table, outs = r.table, []
    for columns in (table.shape[1], 33, 1000):
        r.table = widened(table, columns)
        r.ws = torch.empty(R.riftkv_decode_workspace_size(r.cfg, r.cache, 3, columns), dtype=torch.uint8, device="cuda")
        a, b = r.step(0), r.step(0)
        torch.cuda.synchronize()
        assert int(r.status) == 0 and torch.equal(a, b), columns
        outs.append(a.cpu().double().numpy())
    for o in outs[1:]:
        assert rowwise_rel_err(o, outs[0]) <= GATE
