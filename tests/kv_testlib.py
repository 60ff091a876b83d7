"""Plain float64 forms of the paged key-value cache, for its tests."""
from __future__ import annotations

import math

import torch

LARGEST = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
STORES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn, "int8": torch.int8}


def half_step(dtype):
    """Largest relative error of one rounding."""
    return torch.finfo(dtype).eps / 2


def quantise(x, store):
    """(codes as float64, scale bytes) of rows x, by the definition."""
    f = x.double()
    most = f.abs().amax(-1)
    bad = ~torch.isfinite(f).all(-1)
    most = torch.where(bad, torch.ones_like(most), most)
    byte = torch.ones_like(most, dtype=torch.int64)
    for b in range(1, 254):   # the first that is large enough
        byte = torch.where(most > LARGEST[store] * 2.0 ** (b - 127), torch.full_like(byte, b + 1), byte)
    y = torch.ldexp(torch.where(bad[..., None], torch.zeros_like(f), f), (127 - byte)[..., None].double())
    if store == torch.int8:
        code = torch.round(y)
    else:
        step = torch.ldexp(torch.ones_like(y), (torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4).double())
        code = torch.round(y / step) * step
    return code, torch.where(bad, torch.full_like(byte, 255), byte)


class Pages:
    """A pool of pages on the GPU, every byte of it all ones (NaN, or the scale byte
    255) until written, and a table of shuffled pages."""

    def __init__(self, R, store, n_kv, hd, page, capacity, seed=0, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.page, self.store = page, STORES[store]
        per = [max(1, -(-c // page)) for c in capacity]
        n_pages = sum(per) + spare
        order = torch.randperm(n_pages, generator=g)
        wide = max(per)
        table = torch.full((len(per), wide), -7, dtype=torch.int32)   # unused entries are never read
        at = 0
        for i, p in enumerate(per):
            table[i, :p] = order[at:at + p].int()
            at += p
        self.table = table.cuda()
        size = torch.empty((), dtype=self.store).element_size()
        shape = (n_pages, n_kv, page, hd)
        mk = lambda: torch.full((*shape[:3], hd * size), 255, dtype=torch.uint8, device="cuda").view(self.store)
        self.k, self.v = mk(), mk()
        self.ks = self.vs = None
        if self.store in LARGEST:
            self.ks = torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda")
            self.vs = torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda")
        self.cache = R.riftkv_cache(self.k, self.v, self.ks, self.vs)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def put(self, R, seq, k, v, first=0):
        """Rows of one sequence through riftkv_write."""
        n = k.shape[0]
        if n:
            ids = torch.full((n,), seq, dtype=torch.int32, device="cuda")
            pos = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
            R.riftkv_write(self.cache, k, v, self.table, pos, self.status, seq_ids=ids)

    def rows(self, seq, n):
        """The values (float64, on the CPU) of the first n rows of a sequence: k, v [n][n_kv][hd]."""
        pages = self.table[seq, :-(-n // self.page)].long().cpu()
        out = []
        for x, s in ((self.k, self.ks), (self.v, self.vs)):
            y = x.view(torch.uint8).cpu()[pages].view(self.store).to(torch.float32).double()
            if s is not None:
                b = s.cpu()[pages].double()
                y = y * torch.where(b == 255, torch.full_like(b, math.nan), torch.ldexp(torch.ones_like(b), b - 127))[..., None]
            out.append(y.transpose(1, 2).flatten(0, 1)[:n])
        return out


def attend(q, k, v, scale):
    """float64 attention of q [heads][hd] over k, v [n][n_kv][hd], and what its float32
    evaluation may be off by, before the output's own rounding."""
    heads, hd = q.shape
    n, n_kv = k.shape[:2]
    if n == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    g = heads // n_kv
    kk, vv = k.repeat_interleave(g, 1).transpose(0, 1), v.repeat_interleave(g, 1).transpose(0, 1)   # [heads][n][hd]
    s = (kk @ q[:, :, None])[..., 0] * scale
    w = torch.softmax(s, -1)
    o = (w[:, None] @ vv)[:, 0]
    # a score: hd products summed in float32, scaled twice; a weight: twice its score's error and an exponential of 2^-22;
    # the sums over n weights
    e_score = (hd + 4) * 2.0 ** -24 * ((kk.abs() @ q.abs()[:, :, None])[..., 0] * abs(scale)).amax(-1)
    rel = 2 * e_score + 2.0 ** -21 + (n + 8) * 2.0 ** -24
    return o, rel[:, None] * (w[:, None] @ vv.abs())[:, 0]
