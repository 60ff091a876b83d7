"""The paged key-value cache's C ABI on the CPU: exports, argument checks,
frequencies.  No kernel is launched: every call below returns before any HIP call."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # a non-NULL, aligned value; never dereferenced


@pytest.fixture(scope="module")
def R():
    import paper_2609_29029_amd as R
    if not R.lib_available():
        from paper_2609_29029_amd.build import build
        build()
    R.load()
    return R


@pytest.fixture(scope="module")
def L(R):
    from paper_2609_29029_amd import kv
    return kv._load()


def cache(**over):
    from paper_2609_29029_amd import kv
    a = dict(k=FAKE, v=FAKE, ks=FAKE, vs=FAKE, n_pages=8, page=16, heads=4, hd=128, dt=2, **{})
    a.update(over)
    return kv._CacheStruct(a["k"], a["v"], a["ks"], a["vs"], a["n_pages"], a["page"], a["heads"], a["hd"], a["dt"])


BAD_CACHES = [(dict(k=None), 1), (dict(vs=None), 1), (dict(dt=4), 3), (dict(dt=-1), 3), (dict(page=8), 2),
              (dict(page=24), 2), (dict(page=8192), 2), (dict(n_pages=0), 2), (dict(n_pages=1 << 27), 2),
              (dict(heads=0), 2), (dict(heads=1025), 2), (dict(hd=0), 2), (dict(hd=96), 8), (dict(v=FAKE + 8), 2),
              (dict(ks=FAKE + 4), 2)]


def test_exports(R, L):
    with open(os.path.join(ROOT, "include", "rift_kv.h")) as f:
        names = re.findall(r"RIFT_API\s+[\w\s\*]+?\b(riftkv_\w+)\s*\(", f.read())
    assert tuple(names) == R.KV_EXPORTS
    for n in names:
        assert hasattr(L, n), n
    assert L.riftkv_abi_version() == 1


@pytest.mark.parametrize("name", ["riftkv_write", "riftkv_read"])
def test_rows_are_checked(L, name):
    base = dict(cache=None, k=FAKE, ldk=512, v=FAKE, ldv=512, dt=1, table=FAKE, n_seq=4, pages=2, ids=None, pos=FAKE,
                rows=5, status=FAKE)

    def call(c=None, **over):
        a = dict(base, **over)
        c = cache() if c is None else c
        return getattr(L, name)(ctypes.byref(c), a["k"], a["ldk"], a["v"], a["ldv"], a["dt"], a["table"], a["n_seq"],
                                a["pages"], a["ids"], a["pos"], a["rows"], a["status"], None)

    for over, status in BAD_CACHES:
        assert call(cache(**over)) == status, over
    assert getattr(L, name)(None, FAKE, 512, FAKE, 512, 1, FAKE, 4, 2, None, FAKE, 5, FAKE, None) == 1
    for over in (dict(k=None), dict(v=None), dict(table=None), dict(pos=None), dict(status=None)):
        assert call(**over) == 1, over
    for over in (dict(rows=-1), dict(n_seq=-1), dict(pages=-1), dict(pages=1 << 27), dict(pages=(1 << 26) + 1), dict(ldk=511), dict(ldv=508),
                 dict(ldk=516), dict(k=FAKE + 2)):
        assert call(**over) == 2, over
    assert call(dt=2) == 3
    assert call(dt=0, ldk=514) == 2
    assert call(rows=(1 << 29) + 1) == 8
    assert call(rows=0, k=None, v=None, table=None, pos=None) == 0      # nothing to do
    if name == "riftkv_write":
        assert call(cache(dt=0, ks=None, vs=None)) == 3                 # bf16 rows in f32 pages


def test_attention_is_checked(L):
    base = dict(q=FAKE, ldq=1024, heads=8, dt=1, table=FAKE, n_seq=4, pages=2, lens=FAKE, scale=0.1, out=FAKE, ldo=1024,
                status=FAKE, ws=FAKE, wsb=1 << 30)

    def call(c=None, **over):
        a = dict(base, **over)
        c = cache() if c is None else c
        return L.riftkv_attention(ctypes.byref(c), a["q"], a["ldq"], a["heads"], a["dt"], a["table"], a["n_seq"],
                                  a["pages"], a["lens"], a["scale"], a["out"], a["ldo"], a["status"], a["ws"], a["wsb"],
                                  None)

    for over, status in BAD_CACHES:
        assert call(cache(**over)) == status, over
    for over in (dict(q=None), dict(out=None), dict(lens=None), dict(table=None), dict(status=None), dict(ws=None)):
        assert call(**over) == 1, over
    for over in (dict(heads=6), dict(heads=0), dict(heads=4100), dict(n_seq=-1), dict(n_seq=65536), dict(pages=-1),
                 dict(pages=1 << 27), dict(pages=(1 << 26) + 1), dict(ldq=1016), dict(ldo=1028), dict(out=FAKE + 8)):
        assert call(**over) == 2, over
    assert call(dt=3) == 3
    assert call(cache(dt=0, ks=None, vs=None)) == 3                     # bf16 queries on f32 pages
    assert call(scale=float("nan")) == 7 and call(scale=float("inf")) == 7
    assert call(n_seq=65535, pages=1 << 26) == 8                        # more tiles than a wave counts
    assert call(ws=FAKE + 16) == 5 and call(wsb=16) == 5
    assert call(n_seq=0, q=None, out=None, lens=None, table=None) == 0


def test_attention_workspace_never_shrinks(L):
    for heads, kv in ((32, 32), (32, 8), (64, 1), (20, 1)):
        for hd in (64, 128):
            c = cache(heads=kv, hd=hd)
            size = lambda n, p: L.riftkv_attention_workspace_size(ctypes.byref(c), heads, n, p)
            last = 0
            for n in (0, 1, 2, 3, 7, 8, 50, 300, 5000, 65535):
                assert size(n, 4) >= last
                last = size(n, 4)
                by_pages = [size(n, p) for p in (0, 1, 2, 5, 100, 20000)]
                assert by_pages == sorted(by_pages)
            assert 256 <= last < 64 << 20
    c = cache()
    assert L.riftkv_attention_workspace_size(ctypes.byref(c), 6, 1, 1) == 0
    assert L.riftkv_attention_workspace_size(ctypes.byref(c), 8, -1, 1) == 0


def test_rope_is_checked(L):
    f = np.ones(64)
    base = dict(q=FAKE, ldq=512, nq=4, qo=FAKE, ldqo=512, k=FAKE, ldk=256, nk=2, ko=FAKE, ldko=256, dt=1, pos=FAKE,
                rows=3, hd=128, rot=128, layout=0, f=f, mag=1.0)

    def call(**over):
        a = dict(base, **over)
        return L.riftkv_rope(a["q"], a["ldq"], a["nq"], a["qo"], a["ldqo"], a["k"], a["ldk"], a["nk"], a["ko"], a["ldko"],
                             a["dt"], a["pos"], a["rows"], a["hd"], a["rot"], a["layout"],
                             None if a["f"] is None else a["f"].ctypes.data, a["mag"], None)

    for over in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None), dict(f=None)):
        assert call(**over) == 1, over
    for over in (dict(rows=-1), dict(nq=-1), dict(nk=4097), dict(hd=0), dict(hd=257), dict(rot=0), dict(rot=3),
                 dict(hd=64), dict(ldq=511), dict(ldko=255), dict(ldqo=520)):   # the last: in place with another stride
        assert call(**over) == 2, over
    assert call(dt=5) == 3
    assert call(layout=2) == 8
    assert call(f=np.full(64, np.inf)) == 7 and call(mag=float("nan")) == 7
    assert call(rows=0) == 0 and call(nq=0, nk=0, q=None, k=None) == 0
    assert call(rows=1 << 30) == 8


def test_rope_frequencies(R):
    """Against the published formulas, worked out by hand for a few pairs."""
    f, m = R.riftkv_rope_freqs(128)
    assert m == 1.0 and f.shape == (64,)
    assert np.allclose(f, 10000.0 ** (-np.arange(64) / 64.0), rtol=1e-14)
    g, m = R.riftkv_rope_freqs(128, scaling="linear", factor=4.0)
    assert m == 1.0 and np.allclose(g, f / 4, rtol=1e-15)
    g, m = R.riftkv_rope_freqs(128, scaling="base", factor=4.0)
    assert m == 1.0 and g[0] == 1.0 and math.isclose(g[63], f[63] / 4, rel_tol=1e-12)   # the last pair: slowed by the factor
    # ramp: pair 64 ln(4096 / (2 pi n)) / ln 10000 turns n times in 4,096: 20.94 (n = 32), 45.03 (n = 1)
    g, m = R.riftkv_rope_freqs(128, scaling="ramp", factor=8.0, original_len=4096, low=1, high=32)
    assert math.isclose(m, 1 + 0.1 * math.log(8))
    assert np.allclose(g[:21], f[:21], rtol=1e-15) and np.allclose(g[46:], f[46:] / 8, rtol=1e-14)
    r = (30 - 20) / (46 - 20)
    assert math.isclose(g[30], f[30] * (1 - r) + f[30] / 8 * r, rel_tol=1e-13)
    # bands: turns in 8,192 positions at base 500,000
    f5, _ = R.riftkv_rope_freqs(128, base=500000.0)
    g, m = R.riftkv_rope_freqs(128, base=500000.0, scaling="bands", factor=8.0, original_len=8192, low=1, high=4)
    turns = 8192 * f5 / (2 * math.pi)
    assert m == 1.0 and np.allclose(g[turns > 4], f5[turns > 4], rtol=1e-15)
    assert np.allclose(g[turns < 1], f5[turns < 1] / 8, rtol=1e-14)
    mid = (turns >= 1) & (turns <= 4)
    s = (turns[mid] - 1) / 3
    assert mid.sum() >= 5 and np.allclose(g[mid], f5[mid] * s + f5[mid] / 8 * (1 - s), rtol=1e-13)


def test_decode_step_is_checked(R, L):
    layer = R.LayerWeights(*[FAKE] * 9)
    bad_layer = R.LayerWeights(*([FAKE] * 8 + [None]))
    model = dict(d=512, n_heads=4, head_dim=128, ffn=1408, n_layers=1, rms_eps=1e-6, rope_base=1e4, dt_code=R.RIFT_BF16)

    def call(c=None, w=layer, over=None, x=FAKE, table=FAKE, n_seq=3, pages=4, pos=FAKE, out=FAKE, status=FAKE, ws=FAKE,
             wsb=1 << 30):
        cfg = R.model_cfg(**dict(model, **(over or {})))
        return L.riftkv_decode_step(ctypes.byref(cfg), None if w is None else ctypes.byref(w), x,
                                    ctypes.byref(cache() if c is None else c), table, n_seq, pages, pos, out, status, ws,
                                    wsb, None)

    for over, status in BAD_CACHES:
        assert call(cache(**over)) in (status, 2), over      # (other heads than the model's: a shape too)
    for bad in (dict(x=None), dict(w=None), dict(w=bad_layer), dict(table=None), dict(pos=None), dict(out=None),
                dict(status=None), dict(ws=None)):
        assert call(**bad) == 1, bad
    assert call(cache(heads=2)) == 2 and call(cache(hd=64)) == 2
    for bad in (dict(n_seq=-1), dict(n_seq=65536), dict(pages=-1), dict(pages=1 << 27)):
        assert call(**bad) == 2, bad
    assert call(cache(dt=0, ks=None, vs=None)) == 8                       # float32 pages
    assert call(over=dict(dt_code=R.RIFT_F32)) == 8
    assert call(over=dict(d=500)) == 2
    assert call(ws=FAKE + 16) == 5 and call(wsb=4096) == 5
    assert call(n_seq=0) == 0 and call(over=dict(n_layers=0)) == 0
    cfg = R.model_cfg(**model)
    c = cache()
    size = lambda n, p: L.riftkv_decode_workspace_size(ctypes.byref(cfg), ctypes.byref(c), n, p)
    assert size(-1, 4) == 0 and size(4, -1) == 0
    sizes = [size(n, 64) for n in (0, 1, 2, 9, 60, 700, 5000)]
    assert sizes == sorted(sizes) and size(9, 64) <= size(9, 640)


@pytest.mark.parametrize("over, status", [
    (dict(rotary_dim=0), 2), (dict(rotary_dim=7), 2), (dict(rotary_dim=258), 2), (dict(base=1.0), 7),
    (dict(base=float("inf")), 7), (dict(scaling="linear", factor=0.5), 7), (dict(scaling="linear", factor=float("nan")), 7),
    (dict(scaling="base", factor=2.0, rotary_dim=2), 2), (dict(scaling="ramp", factor=2.0), 7),
    (dict(scaling="bands", factor=2.0, original_len=4096, low=4, high=1), 7)])
def test_rope_frequencies_are_checked(R, over, status):
    with pytest.raises(R.RiftError) as e:
        R.riftkv_rope_freqs(**dict(dict(rotary_dim=64), **over))
    assert e.value.status == status


def test_python_checks(R):
    """Shapes, types and places that the wrappers refuse before the C ABI."""
    torch = pytest.importorskip("torch")
    z = torch.zeros(2, 4, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        R.riftkv_cache(z, z)                                   # not on a GPU
    with pytest.raises(ValueError):
        R.riftkv_rope(None, None, None, np.ones(4))
    with pytest.raises(ValueError):
        R.riftkv_rope_freqs(64, scaling="unknown")
