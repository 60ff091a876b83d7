"""Numbers that 32 bits do not hold are refused by the Python calls of the paged cache, not cut off on their way to the C ABI."""
from types import SimpleNamespace as Stub

import pytest

from tests.test_kv_cpu import L, R  # noqa: F401  (fixtures)

PAST = (1 << 32, (1 << 32) + 5, 1 << 31, -(1 << 32), -(1 << 31) - 1)


@pytest.fixture
def pages(R):  # noqa: F811
    torch = pytest.importorskip("torch")
    kv = __import__("paper_2609_29029_amd.kv", fromlist=["kv"])
    kv._load()
    c = kv.KvCache.__new__(kv.KvCache)
    c.device, c.dt, c.n_layers, c.n_pages, c.n_kv_heads, c.page_size, c.head_dim = 0, kv.RIFTKV_BF16, 1, 8, 2, 16, 64
    c.struct = kv._CacheStruct(None, None, None, None, 8, 16, 2, 64, kv.RIFTKV_BF16)
    c.ref = kv.ctypes.byref(c.struct)
    return torch, c


@pytest.mark.parametrize("x", PAST)
def test_numbers(R, pages, x):  # noqa: F811
    torch, c = pages
    none = Stub(dtype=torch.bfloat16, shape=(1, 2, 64))
    table = Stub(shape=(1, 4))
    for name in ("keep_first", "keep_last"):
        with pytest.raises(ValueError, match=name):
            R.riftkv_select_pages(c, None, none, table, None, None, None, None, **{name: x})
    with pytest.raises(ValueError, match="prefix_len"):
        R.riftkv_attention_shared(c, none, None, x, table, None, None, None, None)
    with pytest.raises(ValueError, match="rotary_dim"):
        R.riftkv_rope_freqs(x)
    sizes = {R.riftkv_attention_workspace_size: (1, 2, 4), R.riftkv_attention_shared_workspace_size: (1, 2, 3, 4),
             R.riftkv_select_pages_workspace_size: (1, 4), R.riftkv_attention_pages_workspace_size: (1, 2, 3)}
    for size, good in sizes.items():
        assert size(c, *good) > 0
        for i in range(len(good)):
            with pytest.raises(ValueError, match="32 bits"):
                size(c, *good[:i], x, *good[i + 1:])
    with pytest.raises(ValueError, match="32 bits"):
        R.riftkv_decode_workspace_size(R.ModelCfg(), c, x, 4)


@pytest.mark.parametrize("x", PAST[:3])
def test_shapes(R, pages, x):  # noqa: F811
    torch, c = pages

    def q(*shape):
        return Stub(dtype=torch.bfloat16, shape=shape, dim=lambda: len(shape), get_device=lambda: 0)

    calls = [lambda t, y: R.riftkv_attention(c, y, t, None, None, None, None),
             lambda t, y: R.riftkv_attention_shared(c, y, None, 0, t, None, None, None, None),
             lambda t, y: R.riftkv_select_pages(c, None, y, t, None, None, None, None),
             lambda t, y: R.riftkv_attention_pages(c, y, t, None, None, None, None, None)]
    for call in calls:
        for t, y in (((x, 4), q(x, 2, 64)), ((1, x), q(1, 2, 64)), ((1, 4), q(1, x, 64))):
            with pytest.raises(ValueError, match="31 bits"):
                call(Stub(shape=t), y)
    for t, y in (((x, 4), q(1, 2, 64)), ((1, x), q(1, 2, 64)), ((1, 4), q(x, 2, 64))):
        for move in (lambda: R.riftkv_write(c, y, y, Stub(shape=t), None, None), lambda: R.riftkv_read(c, Stub(shape=t), None, y, y, None)):
            with pytest.raises(ValueError, match="31 bits"):
                move()
    for t in ((x, 4), (1, x)):
        with pytest.raises(ValueError, match="31 bits"):
            R.riftkv_page_bounds(c, None, Stub(shape=t), None, None)
    for shape in ((x, 2, 64), (2, x, 64), (2, 2, x)):
        with pytest.raises(ValueError, match="31 bits"):
            R.riftkv_rope(q(*shape), None, None, None)
