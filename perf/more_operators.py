"""Operators of the paged key-value cache for long contexts of images, as cases that can be timed and compared.

axes       rotary positions of several axes (a tile's place in the scene, row and column in the tile): every pair takes
           its angle from one of them (`riftkv_rope_axes`)
shared     one new token of every sequence over a prefix that all share, read once for all, and the sequence's own pages
           (`riftkv_attention_shared`)
bounds     the smallest and largest key value of each element of a page, for new or grown pages (`riftkv_page_bounds`)
select     the pages whose bounds promise the largest scores for a new token, a list for each key head, with the
           first and last pages always in it (`riftkv_select_pages`)
pages      one new token of every sequence over the pages of such lists (`riftkv_attention_pages`)

With `own` false `run` computes them in elementary torch operations in 32 bits (page scores and angles in 64); with
`own` true it makes the package's calls.  Sizes: the LLaMA-7B-shaped decoder's 32 heads of 128 dimensions, the 400-tile
scene's prompts and budgets, and grouped heads, 64-dimensional heads, long contexts and large batches as serving
meets them.

Pages: k, v [n_pages][kv_heads][page][head_dim]; 8-bit pages have a scale byte b a row [n_pages][kv_heads][page], for
2^(b - 127).  Bounds: [n_pages][kv_heads][2][head_dim], the smallest values, then the largest; float32 with float32
pages, else bfloat16.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn, "int8": torch.int8}
BYTES = {"bf16": 2, "f32": 4, "fp8": 1, "int8": 1}
SCALED = ("fp8", "int8")
FIRST, LAST = 1, 2            # pages at a context's two ends that a selection always keeps


# ------------------------------------------------------------------ the cases
def _named(name, c):
    return dict(name=name, **c) if name else c


def _axes(name, tokens, q_heads, k_heads, head_dim, rotary_dim, axes, order, layout, far, type="bf16"):
    return _named(name, dict(op="axes", tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=head_dim,
                             rotary_dim=rotary_dim, axes=axes, order=order, layout=layout, far=far, type=type))


def _shared(name, seqs, prefix, shortest, longest, heads, kv_heads, head_dim, page, store, type="bf16"):
    return _named(name, dict(op="shared", seqs=seqs, prefix=prefix, shortest=shortest, longest=longest, heads=heads,
                             kv_heads=kv_heads, head_dim=head_dim, page=page, store=store, type=type))


def _bounds(name, seqs, shortest, longest, new, kv_heads, head_dim, page, store, type="bf16"):
    return _named(name, dict(op="bounds", seqs=seqs, shortest=shortest, longest=longest, new=new, kv_heads=kv_heads,
                             head_dim=head_dim, page=page, store=store, type=type))


def _sparse(op, name, seqs, shortest, longest, top, heads, kv_heads, head_dim, page, store, type="bf16"):
    return _named(name, dict(op=op, seqs=seqs, shortest=shortest, longest=longest, top=top, heads=heads, kv_heads=kv_heads,
                             head_dim=head_dim, page=page, store=store, type=type))


def listed():
    return [
        # one decode step of the scene's 100 prompts: tile, row and column, where latency counts
        _axes("axes_step", 100, 32, 32, 128, 128, 3, "sections", "half", 400),
        # the scene's retained vision tokens with the text around them, grouped heads, axes in turn, neighbours as pairs
        _axes("axes_scene", 22204, 32, 8, 128, 128, 3, "turns", "interleaved", 4096),
        # a few sequences after a system prompt of some pages: the smallest of its kind
        _shared("shared_few_int8", 4, 2049, 1, 70, 32, 8, 128, 16, "int8"),
        # the scene's 100 prompts of uneven budgets after the 35 system rows
        _shared("shared_scene", 100, 35, 96, 608, 32, 32, 128, 16, "bf16"),
        # a batch of questions about one long context: the largest call
        _shared("shared_long", 64, 32768, 1, 600, 32, 8, 128, 64, "bf16"),
        # one decode step: the pages that the new tokens went to
        _bounds("bounds_step", 64, 100, 32768, 1, 8, 128, 32, "bf16"),
        # all pages of prompts that were just written, e4m3
        _bounds("bounds_prompts_fp8", 12, 3001, 65536, 0, 8, 128, 32, "fp8"),
        # one long context's next token
        _sparse("select", "select_prompt", 1, 32768, 32768, 64, 32, 8, 128, 32, "bf16"),
        # a serving batch, uneven contexts
        _sparse("select", "select_batch", 48, 17, 65001, 128, 32, 8, 128, 32, "bf16"),
        # one long context's next token over its 64 pages a key head: the smallest attention
        _sparse("pages", "pages_prompt", 1, 32768, 32768, 64, 32, 8, 128, 32, "bf16"),
        # a serving batch over e4m3 pages, some contexts shorter than the list
        _sparse("pages", "pages_batch_fp8", 64, 17, 32001, 128, 64, 8, 128, 32, "fp8"),
        # float32 sequences with 64-dimensional heads, a group that is not a power of two
        _sparse("pages", "pages_f32", 24, 0, 20011, 40, 12, 4, 64, 16, "f32", "f32"),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], even over the logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(("axes", "shared", "shared", "bounds", "select", "pages", "pages"))
    head_dim, page = rng.choice((64, 128, 128)), rng.choice((16, 16, 32, 32, 64, 128, 256))
    if op == "axes":
        k_heads = rng.choice((1, 2, 5, 8, 12, 32))
        return _axes(None, _between(rng, 1, 22204), min(32, k_heads * rng.choice((1, 2, 3, 4, 8))), k_heads, head_dim,
                     rng.choice((head_dim, head_dim, head_dim // 2)), rng.choice((2, 3, 4)), rng.choice(("sections", "turns")),
                     rng.choice(("half", "interleaved")), _between(rng, 64, 1 << 20), rng.choice(("bf16", "bf16", "f32")))
    type, store = rng.choice((("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "f32"),
                              ("f32", "fp8"), ("f32", "int8"), ("f32", "bf16")))
    kv_heads = rng.choice((1, 2, 3, 4, 8, 12, 32))
    group = rng.choice((1, 2, 3, 4, 6, 8, 16, 20))
    seqs = _between(rng, 1, 128)
    wide = kv_heads * head_dim
    if op == "shared":
        # products of the whole call, and values of the own pages
        prefix = _between(rng, 1, max(1, min(32768, 6_000_000_000 // (seqs * group * wide * (3 if type == "f32" else 1)))))
        longest = _between(rng, 1, max(1, min(8192, 50_000_000 // (seqs * wide))))
        return _shared(None, seqs, prefix, rng.choice((0, 1, longest // 3, longest)), longest, kv_heads * group, kv_heads,
                       head_dim, page, store, type)
    most = (300_000_000 if op == "bounds" else 400_000_000) // BYTES[store]   # values of the keys
    least = 64 * page if op == "select" else 1                                # pages to choose from
    longest = _between(rng, least, max(least, min(131072, most // (seqs * wide))))
    shortest = rng.choice((0, 1, longest // 3, longest))
    if op == "bounds":
        return _bounds(None, seqs, shortest, longest, rng.choice((0, 0, 1, 100)), kv_heads, head_dim, page, store, type)
    top = _between(rng, 8, min(256, 4096 // page, longest // page // 2)) if op == "select" else _between(rng, 4, min(256, 4096 // page))
    return _sparse(op, None, seqs, shortest, longest, top, kv_heads * group, kv_heads, head_dim, page, store, type)


def _lengths(case):
    """Lengths of a case's sequences, evenly spread."""
    n, lo, hi = case["seqs"], case["shortest"], case["longest"]
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _first_new(case, n):
    """The first token of a sequence of n that its bounds do not hold yet; the first page's where `new` is 0."""
    return max(0, n - case["new"]) // case["page"] * case["page"] if case["new"] else 0


def work(case):
    d, t = case["head_dim"], BYTES[case["type"]]
    if case["op"] == "axes":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"]) * d
        return {"bytes": 2 * n * t + 4 * case["tokens"] * case["axes"], "flops": 3 * n * case["rotary_dim"] / d}
    row = d * BYTES[case["store"]] + (case["store"] in SCALED)   # of a head's key or value in the pages
    lens, page, kv = _lengths(case), case["page"], case["kv_heads"]
    bound = 2 * d * (4 if case["store"] == "f32" else 2)          # of a page and key head
    held = [-(-n // page) for n in lens]
    if case["op"] == "bounds":
        new = [n - _first_new(case, n) for n in lens]
        return {"bytes": kv * (sum(new) * row + sum(-(-n // page) for n in new) * bound), "flops": 2 * kv * sum(new) * d}
    tokens = case["seqs"] * case["heads"] * d * t                 # the queries, or the outputs
    if case["op"] == "select":
        return {"bytes": kv * sum(held) * bound + tokens + 4 * case["seqs"] * kv * case["top"],
                "flops": 4 * case["heads"] * sum(held) * d}
    if case["op"] == "shared":
        keys = case["prefix"] + sum(lens)
        return {"bytes": 2 * keys * kv * row + 2 * tokens, "flops": 4 * (case["seqs"] * case["prefix"] + sum(lens)) * case["heads"] * d}
    keys = sum(n if h <= case["top"] else (case["top"] - 1) * page + n - (h - 1) * page for n, h in zip(lens, held))
    return {"bytes": 2 * keys * kv * row + 2 * tokens, "flops": 4 * keys * case["heads"] * d}


# ------------------------------------------------------------------ inputs
def _axis_of(case):
    """The axis of each pair: runs of pairs, the first axis' the shortest, or the axes in turn."""
    pairs, n = case["rotary_dim"] // 2, case["axes"]
    if case["order"] == "turns":
        return [j % n for j in range(pairs)]
    first = pairs // (n + 1)
    return [0 if j < first else 1 + (j - first) * (n - 1) // (pairs - first) for j in range(pairs)]


def _store(g, shape, store):
    """Values of pages, and their scale bytes."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if store == "f32" else torch.bfloat16)
    if store == "fp8":
        x = x.mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn)
    elif store == "int8":
        x = x.mul_(40).round_().clamp_(-127, 127).to(torch.int8)
    return x, torch.randint(118, 122, shape[:3], generator=g, device="cuda", dtype=torch.uint8) if store in SCALED else None


def _tables(g, lens, page, more=0):
    """Number of pages, the table of the sequences' own in any order, and `more` pages besides."""
    held = [max(1, -(-n // page)) for n in lens]
    n_pages = sum(held) + more + 3
    order = torch.randperm(n_pages, generator=g, device="cuda", dtype=torch.int32)
    first = torch.tensor([0] + held, device="cuda").cumsum(0)[:-1]
    at = (first[:, None] + torch.arange(max(held), device="cuda")).clamp_(max=n_pages - 1)   # past a sequence's own: not read
    return n_pages, order[at].contiguous(), order[sum(held):sum(held) + more].contiguous()


def _lists(case, g, lens):
    """Lists as a selection leaves them: both ends of the context, others at random, ascending, -1 behind them."""
    n, kv, top, page = len(lens), case["kv_heads"], case["top"], case["page"]
    held = torch.tensor([-(-x // page) for x in lens], device="cuda")[:, None, None]
    wide = max(top, max(1, -(-max(lens) // page)))
    at = torch.arange(wide, device="cuda")
    rank = torch.rand((n, kv, wide), generator=g, device="cuda")
    rank = torch.where((at < FIRST) | (at >= held - LAST), -1.0, rank)
    rank = torch.where(at < held, rank, 2.0)
    pick = rank.argsort(-1)[..., :top]
    pick = torch.where(pick < held, pick, wide).sort(-1).values
    return torch.where(pick < wide, pick, -1).int().contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    type, d, op = TYPES[case["type"]], case["head_dim"], case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=type)

    if op == "axes":
        T, hq, hk, rotary = case["tokens"], case["q_heads"], case["k_heads"], case["rotary_dim"]
        qkv = normal(T, (hq + 2 * hk) * d)   # a projection's row: queries, keys, values
        freqs, axis = [10000.0 ** (-2.0 * j / rotary) for j in range(rotary // 2)], _axis_of(case)
        return {"op": op, "q": qkv[:, :hq * d].view(T, hq, d), "k": qkv[:, hq * d:(hq + hk) * d].view(T, hk, d),
                "positions": torch.randint(0, case["far"], (case["axes"], T), generator=g, device="cuda", dtype=torch.int32),
                "freqs": torch.tensor(freqs, device="cuda", dtype=torch.float64), "freqs_host": np.array(freqs),
                "axis": torch.tensor(axis, device="cuda"), "axis_host": np.array(axis, dtype=np.int32), "layout": case["layout"],
                "q_out": torch.empty(T, hq, d, device="cuda", dtype=type), "k_out": torch.empty(T, hk, d, device="cuda", dtype=type)}
    lens, page, kv, store = _lengths(case), case["page"], case["kv_heads"], case["store"]
    order = torch.randperm(len(lens), generator=g, device="cuda").tolist()
    lens = [lens[i] for i in order]
    n_pages, table, prefix = _tables(g, lens, page, -(-case["prefix"] // page) if op == "shared" else 0)
    s = {"op": op, "page_table": table, "page": page, "store": store, "kv_heads": kv,
         "lens": torch.tensor(lens, device="cuda", dtype=torch.int32)}
    shape = (n_pages, kv, page, d)
    if op in ("bounds", "select"):
        kind = torch.float32 if store == "f32" else torch.bfloat16
        a, b = (torch.randn((n_pages, kv, 1, d), generator=g, device="cuda", dtype=kind) * 0.45 for _ in range(2))
        top = math.sqrt(2 * math.log(page))   # of as many normal values
        s["bounds"] = torch.cat((torch.minimum(a - top, b), torch.maximum(a, b + top)), 2).contiguous()
    if op != "select" or own:
        s["k"], s["k_scale"] = _store(g, shape, store) if op != "select" else (torch.empty(shape, device="cuda", dtype=TYPES[store]), None)
        if op in ("shared", "pages"):
            s["v"], s["v_scale"] = _store(g, shape, store)
    if op != "bounds":
        s["q"] = normal(len(lens), case["heads"], d).mul_(2)
    if op == "bounds":
        s["begins"] = torch.tensor([_first_new(case, n) for n in lens], device="cuda", dtype=torch.int32)
    if op == "select":
        s["pages"] = torch.empty(len(lens), kv, case["top"], device="cuda", dtype=torch.int32)
    if op == "pages":
        s["pages"] = _lists(case, g, lens)
    if op == "shared":
        s["prefix_table"], s["prefix"] = prefix, case["prefix"]
    if op in ("shared", "pages"):
        s["out"] = torch.empty_like(s["q"])
    if own:   # the cache's handle, and the workspace, that a program keeps
        import paper_2609_29029_amd as R
        scale = torch.empty(shape[:3], device="cuda", dtype=torch.uint8) if store in SCALED and op in ("bounds", "select") else None
        s["cache"] = R.riftkv_cache(s["k"], s.get("v", s["k"]), scale if op == "select" else s["k_scale"], s.get("v_scale", scale))
        s["status"] = torch.zeros(1, device="cuda", dtype=torch.int32)
        size = 0
        if op == "shared":
            size = R.riftkv_attention_shared_workspace_size(s["cache"], *s["q"].shape[:2], s["prefix"], table.shape[1])
        elif op == "select":
            size = R.riftkv_select_pages_workspace_size(s["cache"], len(lens), table.shape[1])
        elif op == "pages":
            size = R.riftkv_attention_pages_workspace_size(s["cache"], *s["q"].shape[:2], case["top"])
        s["workspace"] = torch.empty(max(256, size), device="cuda", dtype=torch.uint8)
    return s


# ------------------------------------------------------------------ plain forms
def _plain_axes(s):
    angle = s["positions"][s["axis"]].double().t() * s["freqs"]   # [T][pairs], in 64 bits: far positions
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = s["freqs"].numel()

    def turn(x, out):
        f = x.float()
        a, b = (f[..., :half], f[..., half:2 * half]) if s["layout"] == "half" else (f[..., :2 * half:2], f[..., 1:2 * half:2])
        y = (a * c - b * n, b * c + a * n)
        y = torch.cat(y, -1) if s["layout"] == "half" else torch.stack(y, -1).flatten(-2)
        return out.copy_(torch.cat((y, f[..., 2 * half:]), -1))

    return {"q": turn(s["q"], s["q_out"]), "k": turn(s["k"], s["k_out"])}


def _power(byte):
    """2^(byte - 127), exact, from the bits of a float32."""
    return (byte.int() << 23).view(torch.float32)


def _rows(s, name, page, head=None):
    """Values [*page.shape][kv_heads][page][head_dim] of pages in 32 bits; with `head` those of one key head each."""
    x, at = s[name], (page,) if head is None else (page, head)
    f = (x.view(torch.uint8)[at].view(x.dtype) if s["store"] in SCALED else x[at]).float()
    return f if s[name + "_scale"] is None else f * _power(s[name + "_scale"][at])[..., None]


def _softmax_parts(q, k, v, there):
    """Largest score, sum of weights and weighted values of q [..][g][d] over k, v [..][n][d] where `there`."""
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1])
    score = score.masked_fill_(~there, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    weight = torch.exp(score.sub_(top))
    return top, weight.sum(-1, keepdim=True), torch.matmul(weight, v)


def _plain_shared(s):
    n, heads, d = s["q"].shape
    kv, P, wide = s["kv_heads"], s["prefix"], s["page_table"].shape[1] * s["page"]
    q = s["q"].float().view(n, kv, -1, d)
    group = q.shape[2]
    # the prefix: the rows of all sequences together
    k, v = (_rows(s, x, s["prefix_table"].long()).transpose(0, 1).reshape(kv, -1, d)[:, :P] for x in ("k", "v"))
    rows = q.transpose(0, 1).reshape(kv, n * group, d)
    m1, l1, o1 = (x.view(kv, n, group, -1).transpose(0, 1)
                  for x in _softmax_parts(rows, k, v.contiguous(), torch.ones(1, dtype=torch.bool, device="cuda")))
    # the sequences' own
    k, v = (_rows(s, x, s["page_table"].long()).transpose(1, 2).reshape(n, kv, wide, d) for x in ("k", "v"))
    there = (torch.arange(wide, device="cuda") < s["lens"][:, None])[:, None, None]
    m2, l2, o2 = _softmax_parts(q, k, v.masked_fill_(~there.transpose(2, 3), 0.0), there)
    m = torch.maximum(m1, m2)
    a, b = torch.exp(m1 - m), torch.exp(m2 - m)
    return s["out"].copy_(((a * o1 + b * o2) / (a * l1 + b * l2)).reshape(n, heads, d))


def _held(s):
    """Pages that each sequence holds."""
    return (s["lens"].long() + s["page"] - 1) // s["page"]


def _plain_bounds(s):
    """Sequence and place of every page with a new token, then their keys all at once."""
    page, wide = s["page"], s["page_table"].shape[1]
    at = torch.arange(wide, device="cuda")
    seq, place = torch.nonzero((at >= s["begins"].long()[:, None] // page) & (at < _held(s)[:, None]), as_tuple=True)
    which = s["page_table"][seq, place].long()
    x = _rows(s, "k", which)
    there = (torch.arange(page, device="cuda") + place[:, None] * page < s["lens"].long()[seq][:, None])[:, None, :, None]
    low, high = x.masked_fill(~there, math.inf).amin(2), x.masked_fill(~there, -math.inf).amax(2)
    s["bounds"][which] = torch.stack((low, high), 2).to(s["bounds"].dtype)
    return s["bounds"]


def _plain_select(s):
    """Scores in 64 bits, a key head at a time; the ends above every score, pages that are not there below."""
    n, heads, d = s["q"].shape
    wide, kv, top = s["page_table"].shape[1], s["kv_heads"], s["pages"].shape[2]
    q = s["q"].double().view(n, kv, -1, d)
    table, held, at = s["page_table"].long(), _held(s)[:, None], torch.arange(wide, device="cuda")
    for h in range(kv):
        b = s["bounds"][:, h][table].double()                                             # [n][wide][2][d]
        x = torch.cat((q[:, h].clamp(max=0), q[:, h].clamp(min=0)), -1).transpose(1, 2).contiguous()   # [n][2 d][group]
        score = torch.matmul(b.flatten(2), x).amax(-1)
        score = torch.where((at < FIRST) | (at >= held - LAST), math.inf, score)
        score = torch.where(at < held, score, -math.inf)
        pick = score.sort(dim=-1, descending=True, stable=True).indices[:, :top]
        pick = torch.where(pick < held, pick, wide).sort(-1).values
        s["pages"][:, h] = -1
        s["pages"][:, h, :pick.shape[1]] = torch.where(pick < wide, pick, -1)
    return s["pages"]


def _plain_pages(s):
    n, heads, d = s["q"].shape
    kv, page, top = s["kv_heads"], s["page"], s["pages"].shape[2]
    place = s["pages"].long()                                                             # [n][kv][top]
    known = place.clamp(min=0)
    which = s["page_table"].long().gather(1, known.flatten(1)).view(n, kv, top)
    head = torch.arange(kv, device="cuda")[:, None].expand(n, kv, top)
    there = (known[..., None] * page + torch.arange(page, device="cuda") < s["lens"].long()[:, None, None, None]) & (place >= 0)[..., None]
    there = there.view(n, kv, top * page)
    k, v = (_rows(s, x, which, head).view(n, kv, top * page, d) for x in ("k", "v"))
    _, l, o = _softmax_parts(s["q"].float().view(n, kv, -1, d), k, v.masked_fill_(~there[..., None], 0.0), there[:, :, None])
    o = torch.where(there.any(-1)[..., None, None], o / l, 0.0)
    return s["out"].copy_(o.reshape(n, heads, d))


# ------------------------------------------------------------------ the package's calls
def _own(s):
    import paper_2609_29029_amd as R
    op = s["op"]
    if op == "axes":
        R.riftkv_rope_axes(s["q"], s["k"], s["positions"], s["freqs_host"], s["axis_host"], s["q_out"], s["k_out"], layout=s["layout"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "shared":
        R.riftkv_attention_shared(s["cache"], s["q"], s["prefix_table"], s["prefix"], s["page_table"], s["lens"], s["out"],
                                  s["workspace"], s["status"])
        return s["out"]
    if op == "bounds":
        R.riftkv_page_bounds(s["cache"], s["bounds"], s["page_table"], s["lens"], s["status"], begins=s["begins"])
        return s["bounds"]
    if op == "select":
        R.riftkv_select_pages(s["cache"], s["bounds"], s["q"], s["page_table"], s["lens"], s["pages"], s["workspace"], s["status"],
                              keep_first=FIRST, keep_last=LAST)
        return s["pages"]
    R.riftkv_attention_pages(s["cache"], s["q"], s["page_table"], s["lens"], s["pages"], s["out"], s["workspace"], s["status"])
    return s["out"]


PLAIN = {"axes": _plain_axes, "shared": _plain_shared, "bounds": _plain_bounds, "select": _plain_select, "pages": _plain_pages}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ------------------------------------------------------------------ in 64 bits
def _exact_axes(s):
    """Pairs as complex numbers, turned by exp(i position frequency), an axis at a time."""
    half, out = s["freqs"].numel(), {}
    for name in ("q", "k"):
        y = s[name].double()
        pairs = y[..., :2 * half].unflatten(-1, (2, half)).transpose(-1, -2) if s["layout"] == "half" else y[..., :2 * half].unflatten(-1, (half, 2))
        z = torch.view_as_complex(pairs.contiguous())
        for axis in range(s["positions"].shape[0]):
            mine = torch.nonzero(s["axis"] == axis)[:, 0]
            a = torch.outer(s["positions"][axis].double(), s["freqs"][mine])
            z[..., mine] *= torch.polar(torch.ones_like(a), a)[:, None]
        z = torch.view_as_real(z)
        y[..., :2 * half] = (z.transpose(-1, -2) if s["layout"] == "half" else z).flatten(-2)
        out[name] = y
    return out


def _exact_value(s, name, page, head):
    """Values of one key head of pages, in 64 bits."""
    x = s[name].view(torch.uint8)[page, head].view(s[name].dtype) if s["store"] in SCALED else s[name][page, head]
    if s[name + "_scale"] is None:
        return x.double()
    return x.double() * (s[name + "_scale"][page, head].long() + (1023 - 127) << 52).view(torch.float64)[..., None]   # (the power function's last bit is not exact)


def _exact_shared(s):
    """A sequence and key head at a time, over the prefix and its own rows as one context; a prefix head is widened once."""
    out = torch.zeros(s["q"].shape, device="cuda", dtype=torch.float64)
    n, heads, d = out.shape
    group, lens, page = heads // s["kv_heads"], s["lens"].tolist(), s["page"]
    for h in range(s["kv_heads"]):
        front = [_exact_value(s, x, s["prefix_table"].long(), h).flatten(0, 1)[:s["prefix"]] for x in ("k", "v")]
        for i in range(n):
            own_pages = s["page_table"][i, :-(-lens[i] // page)].long()
            k, v = (torch.cat((f, _exact_value(s, x, own_pages, h).flatten(0, 1)[:lens[i]])) for f, x in zip(front, ("k", "v")))
            q = s["q"][i, h * group:(h + 1) * group].double()
            out[i, h * group:(h + 1) * group] = torch.softmax(q @ k.t() * d ** -0.5, -1) @ v
    return out


def _exact_bounds(s):
    """A sequence at a time."""
    y, page = s["bounds"].double(), s["page"]
    for i, (b, n) in enumerate(zip(s["begins"].tolist(), s["lens"].tolist())):
        for p0 in range(b // page, -(-n // page), 256):   # some pages at a time, the last one short
            which = s["page_table"][i, p0:min(p0 + 256, -(-n // page))].long()
            for h in range(s["kv_heads"]):
                x = _exact_value(s, "k", which, h)
                y[which, h, 0], y[which, h, 1] = x.min(1).values, x.max(1).values
            if n - (p0 + which.numel()) * page < 0:
                short = _exact_value(s, "k", which[-1:].expand(s["kv_heads"]), torch.arange(s["kv_heads"], device="cuda"))[:, :n - (p0 + which.numel() - 1) * page]
                y[which[-1], :, 0], y[which[-1], :, 1] = short.min(1).values, short.max(1).values
    return y


def _exact_select(s):
    """The definition, a sequence and key head at a time; ranked on the host by (score, lowest page)."""
    out = np.full(s["pages"].shape, -1, dtype=np.int32)
    n, kv, top = out.shape
    group = s["q"].shape[1] // kv
    held = _held(s).tolist()
    for i in range(n):
        ends = [p for p in range(held[i]) if p < FIRST or p >= held[i] - LAST]
        for h in range(kv):
            b = s["bounds"][s["page_table"][i, :held[i]].long(), h].double()
            q = s["q"][i, h * group:(h + 1) * group].double()
            score = torch.stack([torch.where(x < 0, b[:, 0], b[:, 1]).mul(x).sum(-1) for x in q]).amax(0).cpu().numpy()
            order = [int(p) for p in np.lexsort((np.arange(held[i]), -score)) if FIRST <= p < held[i] - LAST]
            pick = sorted((ends + order)[:top])
            out[i, h, :len(pick)] = pick
    return torch.from_numpy(out).cuda()


def _exact_pages(s):
    """A sequence and key head at a time, over the tokens of its list, one page after the other."""
    out = torch.zeros(s["q"].shape, device="cuda", dtype=torch.float64)
    n, heads, d = out.shape
    kv, page, lens, lists = s["kv_heads"], s["page"], s["lens"].tolist(), s["pages"].tolist()
    group = heads // kv
    for i in range(n):
        for h in range(kv):
            places = [p for p in lists[i][h] if p >= 0]
            if not places or not lens[i]:
                continue
            which = s["page_table"][i].long()[torch.tensor(places, device="cuda")]
            tokens = torch.cat([torch.arange(p * page, (p + 1) * page) for p in places]) < lens[i]
            k, v = (_exact_value(s, x, which, h).flatten(0, 1)[tokens.cuda()] for x in ("k", "v"))
            q = s["q"][i, h * group:(h + 1) * group].double()
            out[i, h * group:(h + 1) * group] = torch.softmax(q @ k.t() * d ** -0.5, -1) @ v
    return out


def exact(case, seed):
    return {"axes": _exact_axes, "shared": _exact_shared, "bounds": _exact_bounds, "select": _exact_select,
            "pages": _exact_pages}[case["op"]](prepare(case, seed))
