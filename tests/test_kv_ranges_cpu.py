"""Argument checks of the calls for long contexts on the CPU.  No kernel is launched: every call below returns before any HIP call."""
import ctypes

import numpy as np
import pytest

from tests.test_kv_cpu import BAD_CACHES, FAKE, L, R, cache  # noqa: F401  (fixtures)


def caller(fn, base, order):
    def call(c=None, **over):
        a = dict(base, **over)
        c = cache() if c is None else c
        return fn(ctypes.byref(c), *(a[n] for n in order), None)
    return call


def test_attention_shared_is_checked(L):  # noqa: F811
    base = dict(q=FAKE, ldq=1024, heads=8, dt=1, front=FAKE, prefix=40, table=FAKE, n_seq=4, pages=2, lens=FAKE, scale=0.1, out=FAKE,
                ldo=1024, status=FAKE, ws=FAKE, wsb=1 << 40)
    call = caller(L.riftkv_attention_shared, base, list(base))
    for over, status in BAD_CACHES:
        assert call(cache(**over)) == status, over
    assert L.riftkv_attention_shared(None, *base.values(), None) == 1
    for over in (dict(q=None), dict(out=None), dict(lens=None), dict(table=None), dict(front=None), dict(status=None), dict(ws=None)):
        assert call(**over) == 1, over
    for over in (dict(heads=6), dict(heads=0), dict(heads=4100), dict(n_seq=-1), dict(n_seq=65536), dict(pages=-1), dict(pages=(1 << 26) + 1),
                 dict(ldq=1016), dict(ldo=1028), dict(out=FAKE + 8), dict(q=FAKE + 4), dict(prefix=-1), dict(prefix=(1 << 30) + 1)):
        assert call(**over) == 2, over
    assert call(heads=4096, ldq=1 << 20, ldo=1 << 20, n_seq=(1 << 14) + 1) == 2      # more rows than the prefix' workgroups take
    assert call(dt=3) == 3 and call(cache(dt=0, ks=None, vs=None)) == 3
    assert call(scale=float("nan")) == 7 and call(scale=float("inf")) == 7 and call(scale=3e38) == 7
    assert call(ws=FAKE + 16) == 5 and call(wsb=16) == 5
    assert call(n_seq=0, q=None, out=None, lens=None, table=None, front=None) == 0


def test_attention_pages_is_checked(L):  # noqa: F811
    base = dict(q=FAKE, ldq=1024, heads=8, dt=1, table=FAKE, n_seq=4, pages=2, lens=FAKE, lists=FAKE, top=3, scale=0.1, out=FAKE, ldo=1024,
                status=FAKE, ws=FAKE, wsb=1 << 40)
    call = caller(L.riftkv_attention_pages, base, list(base))
    for over, status in BAD_CACHES:
        assert call(cache(**over)) == status, over
    assert L.riftkv_attention_pages(None, *base.values(), None) == 1
    for over in (dict(q=None), dict(out=None), dict(lens=None), dict(table=None), dict(lists=None), dict(status=None), dict(ws=None)):
        assert call(**over) == 1, over
    for over in (dict(heads=6), dict(heads=0), dict(heads=4100), dict(n_seq=-1), dict(n_seq=65536), dict(pages=-1), dict(pages=(1 << 26) + 1),
                 dict(ldq=1016), dict(ldo=1028), dict(out=FAKE + 8), dict(top=0), dict(top=-1), dict(top=(1 << 20) + 1)):
        assert call(**over) == 2, over
    assert call(cache(page=4096), top=(1 << 18) + 1) == 2               # more than 2^30 tokens
    assert call(dt=3) == 3 and call(cache(dt=0, ks=None, vs=None)) == 3
    assert call(scale=float("nan")) == 7
    assert call(ws=FAKE + 16) == 5 and call(wsb=16) == 5
    assert call(n_seq=0, q=None, out=None, lens=None, table=None, lists=None) == 0


def test_page_bounds_is_checked(L):  # noqa: F811
    base = dict(bounds=FAKE, table=FAKE, n_seq=4, pages=2, begins=FAKE, lens=FAKE, status=FAKE)
    call = caller(L.riftkv_page_bounds, base, list(base))
    for over, status in BAD_CACHES:
        assert call(cache(**over)) == status, over
    assert L.riftkv_page_bounds(None, *base.values(), None) == 1
    for over in (dict(bounds=None), dict(table=None), dict(lens=None), dict(status=None)):
        assert call(**over) == 1, over
    for over in (dict(n_seq=-1), dict(n_seq=65536), dict(pages=-1), dict(pages=(1 << 26) + 1), dict(bounds=FAKE + 8)):
        assert call(**over) == 2, over
    assert call(n_seq=0, bounds=None, table=None, begins=None, lens=None) == 0


def test_select_pages_is_checked(L):  # noqa: F811
    base = dict(bounds=FAKE, q=FAKE, ldq=1024, heads=8, dt=1, table=FAKE, n_seq=4, pages=2, lens=FAKE, first=1, last=1, lists=FAKE, top=3,
                status=FAKE, ws=FAKE, wsb=1 << 40)
    call = caller(L.riftkv_select_pages, base, list(base))
    for over, status in BAD_CACHES:
        assert call(cache(**over)) == status, over
    assert L.riftkv_select_pages(None, *base.values(), None) == 1
    for over in (dict(bounds=None), dict(q=None), dict(lens=None), dict(table=None), dict(lists=None), dict(status=None), dict(ws=None)):
        assert call(**over) == 1, over
    for over in (dict(heads=6), dict(heads=0), dict(n_seq=-1), dict(n_seq=65536), dict(pages=-1), dict(pages=(1 << 26) + 1), dict(ldq=1016),
                 dict(bounds=FAKE + 8), dict(top=0), dict(top=(1 << 20) + 1), dict(first=-1), dict(last=-1), dict(first=2, last=2),
                 dict(first=2 ** 31 - 1, last=2 ** 31 - 1)):
        assert call(**over) == 2, over
    assert call(dt=3) == 3 and call(cache(dt=0, ks=None, vs=None)) == 3
    assert call(ws=FAKE + 16) == 5 and call(wsb=16) == 5
    assert call(n_seq=0, bounds=None, q=None, lens=None, table=None, lists=None) == 0


def test_rope_axes_is_checked(L):  # noqa: F811
    f, x = np.ones(64), (np.arange(64) % 3).astype(np.int32)
    base = dict(q=FAKE, ldq=512, nq=4, qo=FAKE, ldqo=512, k=FAKE, ldk=256, nk=2, ko=FAKE, ldko=256, dt=1, pos=FAKE, n=3, rows=3, hd=128, rot=128,
                layout=0, f=f, x=x, mag=1.0)

    def call(**over):
        a = dict(base, **over)
        a["f"], a["x"] = (None if y is None else y.ctypes.data for y in (a["f"], a["x"]))
        return L.riftkv_rope_axes(*a.values(), None)

    for over in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None), dict(f=None), dict(x=None)):
        assert call(**over) == 1, over
    for over in (dict(rows=-1), dict(nq=-1), dict(nk=4097), dict(hd=0), dict(hd=257), dict(rot=0), dict(rot=3), dict(hd=64), dict(ldq=511),
                 dict(ldko=255), dict(ldqo=520), dict(n=0), dict(n=9), dict(n=-1), dict(n=2), dict(x=x - 1), dict(x=x + 2 ** 30)):
        assert call(**over) == 2, over
    assert call(dt=5) == 3 and call(layout=2) == 8
    assert call(f=np.full(64, np.inf)) == 7 and call(mag=float("nan")) == 7 and call(mag=1e39) == 7
    assert call(rows=0) == 0 and call(nq=0, nk=0, q=None, k=None) == 0
    assert call(rows=1 << 30) == 8


def test_workspaces_never_shrink(L):  # noqa: F811
    for heads, kv in ((32, 32), (32, 8), (64, 1), (20, 1)):
        for hd in (64, 128):
            c = cache(heads=kv, hd=hd)
            r = ctypes.byref(c)
            sizes = (lambda n, p: L.riftkv_attention_shared_workspace_size(r, heads, n, 100, p),
                     lambda n, p: L.riftkv_attention_shared_workspace_size(r, heads, n, p, 100),
                     lambda n, p: L.riftkv_attention_pages_workspace_size(r, heads, n, p + 1),
                     lambda n, p: L.riftkv_select_pages_workspace_size(r, n, p))
            for size in sizes:
                for p in (0, 1, 7, 100, 255, 256, 257, 20000):
                    by_seq = [size(n, p) for n in (0, 1, 2, 3, 5, 7, 8, 9, 16, 31, 33, 50, 64, 65, 100, 127, 128, 129, 300, 5000, 65535)]
                    assert by_seq == sorted(by_seq) and by_seq[0] >= 256
                for n in (1, 3, 20, 64, 1000):
                    by_pages = [size(n, p) for p in (0, 1, 2, 3, 5, 8, 15, 16, 17, 31, 33, 100, 128, 500, 1000, 4000, 20000, 100000)]
                    assert by_pages == sorted(by_pages)
    c = cache()
    for fn, args in ((L.riftkv_attention_shared_workspace_size, (6, 1, 1, 1)), (L.riftkv_attention_shared_workspace_size, (8, -1, 1, 1)),
                     (L.riftkv_attention_shared_workspace_size, (8, 1, -1, 1)), (L.riftkv_attention_shared_workspace_size, (8, 1, 1, -1)),
                     (L.riftkv_attention_pages_workspace_size, (6, 1, 1)), (L.riftkv_attention_pages_workspace_size, (8, 1, 0)),
                     (L.riftkv_select_pages_workspace_size, (-1, 1)), (L.riftkv_select_pages_workspace_size, (1, -1))):
        assert fn(ctypes.byref(c), *args) == 0, args


def test_python_checks(R):  # noqa: F811
    """What the wrappers refuse before the C ABI."""
    torch = pytest.importorskip("torch")
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    f, a = np.ones(32), np.zeros(32, dtype=np.int32)
    pos = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError):
        R.riftkv_rope_axes(x, None, pos, f, a)                  # not on a GPU
    with pytest.raises(ValueError):
        R.riftkv_rope_axes(None, None, pos, f, a)
