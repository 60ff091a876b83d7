"""Plain float64 forms of the attentions over ranges of the paged cache and of the page selection, for their tests."""
from __future__ import annotations

import math

import torch

from tests.kv_testlib import STORES, Pages, attend, half_step

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def randn(seed, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype).cuda()


def filled(R, store, n_kv, hd, page, lens, seed=0, dtype=None, spread=1.0):
    """Pages that hold lens[i] random rows of sequence i; everything else in them is NaN."""
    P = Pages(R, store, n_kv, hd, page, lens, seed=seed)
    dtype = dtype or (torch.float32 if store == "f32" else torch.bfloat16)
    for i, n in enumerate(lens):
        if n:
            kv = randn(seed * 1000 + i, n, 2, n_kv, hd, dtype=dtype, scale=spread)
            P.put(R, i, kv[:, 0], kv[:, 1])
    return P


def check(got, ref, err, dtype, what=""):
    """Within the float32 evaluation's error and the output's own rounding."""
    bound = err + half_step(dtype) * ref.abs() * (1 + 1e-3) + 1e-30
    off = (got.double().cpu() - ref).abs()
    assert bool((off <= bound).all()), f"{what}: {float((off / bound).max())}"


def attend_lists(P, q, lens, lists, scale=None):
    """riftkv_attention_pages: outputs and their errors [n_seq][heads][hd]."""
    n, heads, hd = q.shape
    n_kv = lists.shape[1]
    g = heads // n_kv
    qd = q.double().cpu()
    out, err = torch.zeros_like(qd), torch.zeros_like(qd)
    for i in range(n):
        k, v = P.rows(i, lens[i])
        for h in range(n_kv):
            tokens = [t for p in lists[i, h].tolist() if p >= 0 for t in range(p * P.page, min((p + 1) * P.page, lens[i]))]
            o, e = attend(qd[i, h * g:(h + 1) * g], k[tokens, h:h + 1], v[tokens, h:h + 1], hd ** -0.5 if scale is None else scale)
            out[i, h * g:(h + 1) * g], err[i, h * g:(h + 1) * g] = o, e
    return out, err


def bounds_of(P, seq, n, page):
    """Smallest and largest key values of a page of a sequence of n tokens: [n_kv][2][hd]; NaN where one is."""
    k = P.rows(seq, n)[0][page * P.page:(page + 1) * P.page]
    nan = torch.isnan(k).any(0)
    low, high = (torch.where(nan, math.nan, x) for x in (k.amin(0), k.amax(0)))
    return torch.stack((low, high), 1)


def selection(bounds, table, q, held, n_kv, top, first, last):
    """The definition, by sorting: lists [n_seq][n_kv][top] of float64 scores."""
    n, heads, hd = q.shape
    g = heads // n_kv
    b, qd = bounds.double().cpu(), q.double().cpu()
    out = torch.full((n, n_kv, top), -1, dtype=torch.int32)
    for i in range(n):
        pages = table[i, :held[i]].long().cpu()
        for h in range(n_kv):
            x = qd[i, h * g:(h + 1) * g]
            score = x.clamp(max=0) @ b[pages, h, 0].t() + x.clamp(min=0) @ b[pages, h, 1].t() if held[i] else torch.zeros(g, 0)
            best = [max(c) if not any(s != s for s in c) else -math.inf for c in score.t().tolist()]
            nan = [any(s != s for s in c) for c in score.t().tolist()]
            middle = [p for p in range(held[i]) if first <= p < held[i] - last]
            middle.sort(key=lambda p: (nan[p], -best[p], p))
            ends = [p for p in range(held[i]) if not first <= p < held[i] - last]
            take = sorted((ends + middle)[:top]) if held[i] > top else list(range(held[i]))
            out[i, h, :len(take)] = torch.tensor(take, dtype=torch.int32)
    return out


__all__ = ["STORES", "TYPES", "Pages", "attend", "attend_lists", "bounds_of", "check", "filled", "half_step", "randn", "selection"]
