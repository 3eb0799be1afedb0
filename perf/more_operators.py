"""A paged key-value cache that takes less memory, as cases that can be timed and checked: four bits an element, and fewer keys.

  append     new keys and values go to their slots of pools in microscaled 4-bit floating point (32 elements share a
             power of two), and rows are read back from there
  attention  the new tokens attend their requests' keys in such pools: one token a request, a few, or a prompt's chunk
  weights    what the new tokens' attention weighs each cached key with is added to the key's account, per KV head
  keep       which keys of a request stay: the first, the last, and those with the largest accounts, per KV head
  evict      the keys that stay move to the front of their request's pages, and the pages behind them are free again

`own` selects between the operators' plain forms (elementary torch operations in float32) and the calls of this
library.  Both take what prepare() gives.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "fp8": 1, "mxfp4": 0.53125}     # an element of a pool, its share of a block's scale included

_DEFAULT = {"batch": 1, "q_heads": 32, "kv_heads": 8, "dtype": "bf16", "kv": "", "page": 64, "shortest": 0, "longest": 0,
            "new": 1, "fewest": 0, "sink": 0, "local": 0, "layout": "token", "tokens": 0, "budget": 0, "first": 0, "last": 0}


def _case(name, op, **more):
    c = {"name": name, "op": op}
    c.update({k: v for k, v in more.items() if _DEFAULT[k] != v})
    return c


def _full(case):
    return {**_DEFAULT, **case}


def listed():
    return [
        # the new token of each of 64 requests, stored and read back
        _case("append_b64", "append", kv="mxfp4", tokens=64),
        # a step full of prompt tokens, stored head by head
        _case("append_16k", "append", kv="mxfp4", tokens=16384, page=32, layout="head"),
        # a short conversation of one user: nothing but latency and launches
        _case("decode_2k", "attention", kv="mxfp4", page=16, shortest=2048, longest=2048),
        # a serving batch of 64k contexts
        _case("decode_b16_64k", "attention", kv="mxfp4", batch=16, shortest=65536, longest=65536, page=128, layout="head"),
        # a ragged batch, eight query heads per KV head
        _case("decode_ragged", "attention", kv="mxfp4", batch=48, q_heads=64, page=32, shortest=50, longest=30011),
        # a chunk of a long prompt behind what is cached of it already
        _case("chunk_60k", "attention", kv="mxfp4", shortest=61440, longest=61440, new=2048, fewest=2048),
        # the account of a decoding step, bf16 cache
        _case("weights_b16_32k", "weights", batch=16, shortest=32768, longest=32768),
        # the account of whole prompts, as it stands before the first eviction
        _case("weights_prompt_b4", "weights", batch=4, shortest=1000, longest=4099, new=4099, fewest=4099),
        # one user's 96k tokens go down to a sixth
        _case("keep_96k", "keep", shortest=98304, longest=98304, budget=16384, first=4, last=512),
        # a serving batch whose ragged requests go down to 1000 keys each (some have fewer)
        _case("keep_b64", "keep", batch=64, page=32, shortest=500, longest=9001, budget=1000, first=4, last=64),
        # one user's 32k tokens go down to a quarter
        _case("evict_32k", "evict", shortest=32768, longest=32768, budget=8192, first=4, last=512),
        # a batch that goes back to 4096 keys every 64 steps, quantised pools
        _case("evict_b32", "evict", kv="fp8", batch=32, page=16, shortest=4097, longest=4160, budget=4096, first=4, last=128),
    ]


# (query heads, KV heads)
_HEADS = [(32, 8), (32, 8), (64, 8), (40, 8), (28, 4), (16, 2), (8, 1), (24, 8), (8, 8), (32, 32), (1, 1)]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "weights", "weights", "keep", "evict"])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256])
    hq, hkv = rng.choice(_HEADS)
    dtype, kv = rng.choice([("bf16", ""), ("bf16", "fp8"), ("fp32", ""), ("bf16", "mxfp4")])
    layout = rng.choice(["token", "head"])
    c = dict(q_heads=hq, kv_heads=hkv, page=page, layout=layout)
    if op in ("append", "attention"):
        dtype, kv = "bf16", "mxfp4"
    if op != "keep":
        c.update(dtype=dtype, kv=kv)
    if op == "append":
        c["tokens"] = _between(rng, 1, 16384)
    elif op in ("attention", "weights"):
        kind = rng.choice(["decode", "decode", "few", "prompt"])
        longest = _between(rng, 1, 100000)
        shortest = rng.choice([longest, rng.randint(0, longest), rng.randint(0, longest)])
        new, fewest = {"decode": (1, 1), "few": (rng.randint(2, 8), 1), "prompt": (_between(rng, 16, 4096),) * 2}[kind]
        new = min(new, longest)
        local = rng.choice([0, 0, 0, _between(rng, 16, 8192)])
        c.update(shortest=shortest, longest=longest, new=new, fewest=min(fewest, new), sink=rng.choice([0, 4, 20]) if local else 0, local=local)
        c["batch"] = _between(rng, 1, 128)
    else:
        longest = _between(rng, 16, 100000)
        budget = min(_between(rng, 1, 16384), max(1, longest - rng.choice([1, 64, longest // 2])))
        c.update(shortest=rng.randint(0, longest), longest=longest, budget=budget, first=rng.choice([0, 4, 20]),
                 last=rng.choice([0, 0, 64, _between(rng, 1, 1000)]), batch=_between(rng, 1, 128))
    # no more keys, scores and work than the largest listed cases
    while c.get("batch", 1) > 1 and _too_much({**c, "op": op}):
        c["batch"] = c["batch"] * 2 // 3
    while _too_much({**c, "op": op}):
        c["new"] = c["new"] * 2 // 3
        c["fewest"] = min(c["fewest"], c["new"])
    got = _case("", op, **c)
    del got["name"]
    return got


def _too_much(case):
    c = _full(case)
    if c["op"] == "append":
        return False
    if c["op"] == "keep":
        return c["batch"] * c["longest"] * c["kv_heads"] > 5e6
    if c["op"] == "evict":
        return c["batch"] * c["longest"] * c["kv_heads"] * D > 1.5e8 and c["batch"] > 1
    rows = c["batch"] * c["new"] * c["q_heads"]
    return (rows * c["longest"] > 4.2e9 or c["batch"] * c["longest"] * c["kv_heads"] * D > (1.1e9 if c["op"] == "attention" else 5.4e8)
            or work(c)["flops"] > (2e12 if c["op"] == "attention" else 4e11 if c["dtype"] == "bf16" else 1e11))


# ---- sizes, from the case alone ----------------------------------------------------------------------
def _spread(n, k):
    """n fractions in [0, 1), evenly spread and in no order."""
    return [math.modf((i + 1) * 0.6180339887498949 + 0.381966 * k)[0] for i in range(n)]


def _lengths(c):
    """The requests' lengths: the longest first, the others between, logarithms spread evenly."""
    lo, hi = math.log1p(c["shortest"]), math.log1p(c["longest"])
    return [c["longest"]] + [min(c["longest"], max(c["shortest"], int(round(math.expm1(lo + (hi - lo) * f)))))
                             for f in _spread(c["batch"] - 1, 0)]


def _news(c):
    """The new tokens of the requests (among the lengths)."""
    if c["new"] == 1:
        return [1] * c["batch"]                               # (also where nothing is cached: a row that attends no key)
    if c["fewest"] == c["new"]:
        return [min(n, c["new"]) for n in _lengths(c)]
    return [min(n, max(1, c["fewest"] + int((c["new"] - c["fewest"] + 1) * f))) for n, f in zip(_lengths(c), _spread(c["batch"], 1))]


def _stay(c):
    return [min(n, c["budget"]) for n in _lengths(c)]


def _up(a, b):
    return -(-a // b)


def _attended(c, n, t):
    """Keys that the last t tokens of n attend, over all of them, and keys that at least one of them attends."""
    if not c["local"] or c["local"] + c["sink"] >= n:
        return t * n - t * (t - 1) // 2, n
    w = c["sink"] + c["local"]
    ramp = max(0, min(t, w - (n - t)))                    # tokens that have not w keys yet
    return sum(range(n - t + 1, n - t + ramp + 1)) + (t - ramp) * w, min(n, w + t - 1)


def work(case):
    c = _full(case)
    row, size = c["kv_heads"] * D, _BYTES[c["kv"] or c["dtype"]]
    if c["op"] == "append":
        # rows in, rows of the pool out; those of the pool in, rows out; slots
        return {"bytes": c["tokens"] * (2 * 2 * row * (2 + size) + 16), "flops": 0}
    if c["op"] in ("attention", "weights"):
        pairs, read, tokens = 0, 0, 0
        for n, t in zip(_lengths(c), _news(c)):
            a, k = _attended(c, n, t)
            pairs, read, tokens = pairs + a, read + k, tokens + t
        q = tokens * c["q_heads"] * (D * _BYTES[c["dtype"]] + 4)         # queries and their log-sum-exp
        if c["op"] == "attention":
            return {"bytes": read * 2 * row * size + q + tokens * c["q_heads"] * D * _BYTES[c["dtype"]], "flops": 4 * D * c["q_heads"] * pairs}
        return {"bytes": read * (row * size + 8 * c["kv_heads"]) + q, "flops": 2 * D * c["q_heads"] * pairs}
    keys, stay = sum(_lengths(c)), sum(m for n, m in zip(_lengths(c), _stay(c)) if m < n)
    if c["op"] == "keep":
        return {"bytes": 4 * c["kv_heads"] * (sum(n for n, m in zip(_lengths(c), _stay(c)) if m < n) + stay) + 12 * c["batch"], "flops": 0}
    # keys that move (all but those in front of the first one that goes, about `first`, and where they lie evenly), in and out
    moved = sum(max(0, m - c["first"]) for n, m in zip(_lengths(c), _stay(c)) if m < n)
    read_back = sum(_stay(c)) * row * 2 * (size + 2) if c["kv"] == "mxfp4" else 0
    return {"bytes": moved * c["kv_heads"] * (2 * (2 * D * size + 4) + 4) + read_back + 8 * _up(keys - stay, c["page"]) + 16, "flops": 0}


# ---- microscaled 4-bit floating point ------------------------------------------------------------------
# A row's 128 elements are 64 bytes, element 2 i in the low half of byte i, and four bytes of scales, one for each 32 elements:
# value = (sign, one of 0 0.5 1 1.5 2 3 4 6) * 2^(scale - 127); scale 255: NaN.
def _quantised(x):
    """x [..., 128] float32 -> bytes [..., 64], scales [..., 4]: the least power of two that leaves no element over 6; to nearest, ties to even."""
    x = x.reshape(*x.shape[:-1], 4, 32)
    top = x.abs().amax(-1)
    m, k = torch.frexp(top)
    e = torch.where(m > 0.75, k - 2, k - 3).clamp(min=-127)
    e = torch.where(top > 0, e, -127)
    fine = torch.isfinite(top)
    e = torch.where(fine, e, 0)
    y = torch.ldexp(x.abs().clamp(max=3 * 2.0 ** 126), -e[..., None])
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)).to(torch.uint8)
    code = torch.where(fine[..., None], code + 8 * torch.signbit(x).to(torch.uint8), 0).to(torch.uint8).reshape(*x.shape[:-2], 64, 2)
    return code[..., 0] + 16 * code[..., 1], torch.where(fine, e + 127, 255).to(torch.uint8)


def _values(rows, scales):
    """bytes [..., 64], scales [..., 4] -> [..., 128] float32."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=rows.device)
    table = torch.cat([table, -table])
    x = table[torch.stack([rows & 15, rows >> 4], -1).int()].reshape(*rows.shape[:-1], 4, 32)
    x = torch.ldexp(x, scales.int()[..., None] - 127)
    return torch.where(scales[..., None] == 255, math.nan, x).reshape(*rows.shape[:-1], D)


# ---- inputs ------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 31) + 31)
    return g


def _pool(c, pages, fill, name, s):
    """The pool s[name + "_pages"], [pages, page, kv heads, D], a view in the case's layout, and beside one in four bits its
    scales; fill(shape) gives float32 values (in parts: they are larger), None: zeros."""
    head, four = c["layout"] == "head", c["kv"] == "mxfp4"
    shape = (pages, c["kv_heads"], c["page"]) if head else (pages, c["page"], c["kv_heads"])
    t = torch.zeros(shape + (64 if four else D,), dtype=torch.uint8 if four else _TYPES[c["kv"] or c["dtype"]], device="cuda")
    scales = torch.zeros(shape + (4,), dtype=torch.uint8, device="cuda") if four else None
    part = max(1, (1 << 26) // (c["page"] * c["kv_heads"] * D))
    for a in range(0, pages if fill is not None else 0, part):
        b = min(pages, a + part)
        x = fill((b - a,) + shape[1:] + (D,))
        if four:
            t[a:b], scales[a:b] = _quantised(x)
        else:
            t[a:b] = (50.0 * x).clamp(-448.0, 448.0).to(t.dtype) if c["kv"] == "fp8" else x.to(t.dtype)
    view = (lambda x: x.permute(0, 2, 1, 3)) if head else (lambda x: x)
    s[name + "_pages"] = view(t)
    s[name + "_block"] = view(scales) if four else None


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _table(c, held, n_pages, g):
    count = torch.tensor(held, device="cuda")
    first = count.cumsum(0) - count
    at = torch.arange(max(max(held), 1), device="cuda")
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    return torch.where(at < count[:, None], ids[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous(), ids


def _prepare_append(c, g):
    n = c["tokens"]
    pages = _up(n, c["page"]) + 3
    wide = c["q_heads"] + 2 * c["kv_heads"]                  # the projections of a layer come from one product
    qkv = torch.randn(n, wide, D, generator=g, device="cuda")
    qkv *= torch.exp(0.8 * torch.randn(wide, D, generator=g, device="cuda"))     # some channels are larger than others
    qkv = qkv.to(_TYPES[c["dtype"]])
    i = torch.arange(n, device="cuda")
    ids = torch.randperm(pages, generator=g, device="cuda")
    slots = ids[i // c["page"]] * c["page"] + i % c["page"]
    slots = torch.where(i < n - n // 16, slots, -1)           # (rows behind the step's tokens)
    s = {"k_new": qkv[:, c["q_heads"]:c["q_heads"] + c["kv_heads"]], "v_new": qkv[:, c["q_heads"] + c["kv_heads"]:], "slots": slots}
    _pool(c, pages, None, "k", s)
    _pool(c, pages, None, "v", s)
    # rows read back go where the projections lie (a program has them no more)
    s["back"] = torch.zeros_like(qkv[:, c["q_heads"]:])
    s["k_out"], s["v_out"] = s["back"][:, :c["kv_heads"]], s["back"][:, c["kv_heads"]:]
    s["sizes"] = dict(max_pages=pages, n_pages=pages, max_tokens=n, max_new=n, k_new_strides=s["k_new"].stride()[:2],
                      v_new_strides=s["v_new"].stride()[:2])
    s["back_sizes"] = dict(s["sizes"], k_new_strides=s["k_out"].stride()[:2], v_new_strides=s["v_out"].stride()[:2])
    return s


def _prepare_attention(c, g):
    lens, news = _lengths(c), _news(c)
    held = [_up(n, c["page"]) for n in lens]
    n_pages, tokens = sum(held) + 2, sum(news) + (3 if c["new"] > 1 else 0)
    table, _ = _table(c, held, n_pages, g)
    # keys of a head share an offset, as cached keys do; queries that make a few keys stand out
    shift = torch.randn(c["kv_heads"], D, generator=g, device="cuda")
    near = shift[:, None] if c["layout"] == "head" else shift
    q = (1.5 * torch.randn(tokens, c["q_heads"], D, generator=g, device="cuda")).to(_TYPES[c["dtype"]])
    start = [sum(news[:b]) for b in range(c["batch"] + 1)]
    s = {"q": q, "table": table, "lengths": _int(lens), "token_start": _int(start) if c["new"] > 1 else None, "page": c["page"],
         "new": c["new"], "longest": max(c["longest"], 1), "sink": c["sink"], "local": c["local"], "k_scale": None}
    _pool(c, n_pages, lambda shape: torch.randn(shape, generator=g, device="cuda") + near, "k", s)
    if c["op"] == "attention":
        _pool(c, n_pages, lambda shape: 0.3 + torch.randn(shape, generator=g, device="cuda"), "v", s)
        s["out"], s["lse"] = torch.zeros_like(q), torch.zeros(tokens, c["q_heads"], device="cuda")
    else:
        size = torch.ones(c["kv_heads"], device="cuda")
        if c["kv"] == "fp8":
            s["k_scale"] = 0.01 + 0.02 * torch.rand(c["kv_heads"], generator=g, device="cuda")
            size = 50.0 * s["k_scale"]
        # the attention's log-sum-exp as it comes out for keys so distributed
        row, there, pos = _rows(s)
        count = torch.zeros(tokens + 1, device="cuda")
        seen = (pos + 1).clamp(min=0).float()
        count[row] = seen if not c["local"] else seen.clamp(max=c["sink"] + c["local"])
        by = (size / math.sqrt(D)).repeat_interleave(c["q_heads"] // c["kv_heads"])
        x = q.float() * by[:, None]
        s["lse"] = (x * shift.repeat_interleave(c["q_heads"] // c["kv_heads"], 0)).sum(-1) + x.square().sum(-1) / 2 + count[:tokens, None].log()
        # what earlier steps left in the account, and garbage where keys are new
        s["weights"] = torch.rand(n_pages, c["kv_heads"], c["page"], generator=g, device="cuda")
    s["sizes"] = dict(max_pages=table.shape[1], n_pages=n_pages, max_tokens=max(tokens, 1), max_new=c["new"], n_sink=c["sink"], n_local=c["local"])
    return s


def _accounts(c, pages, g):
    """A few keys have much of the weight; some have none at all, alike to the last bit."""
    w = torch.exp(2.0 * torch.randn(pages, c["kv_heads"], c["page"], generator=g, device="cuda"))
    return torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.05, 0.0, w)


def _prepare_keep(c, g):
    lens = _lengths(c)
    held = [_up(n, c["page"]) for n in lens]
    n_pages = sum(held) + 2
    table, _ = _table(c, held, n_pages, g)
    s = {"weights": _accounts(c, n_pages, g), "table": table, "lengths": _int(lens), "budgets": _int([c["budget"]] * c["batch"]),
         "page": c["page"], "longest": max(c["longest"], 1), "first": c["first"], "last": c["last"],
         "kept": torch.zeros(c["batch"], c["kv_heads"], c["budget"], dtype=torch.int32, device="cuda"),
         "lengths_out": torch.zeros(c["batch"], dtype=torch.int32, device="cuda")}
    s["sizes"] = dict(max_pages=table.shape[1], n_pages=n_pages)
    return s


def _prepare_evict(c, g):
    lens, stay = _lengths(c), _stay(c)
    held = [_up(n, c["page"]) for n in lens]
    n_pages = sum(held) + 40
    table, ids = _table(c, held, n_pages, g)
    n, m = torch.tensor(lens, device="cuda"), torch.tensor(stay, device="cuda")
    # the first, the last and any others, in order; a request that loses none has no list
    i = torch.arange(max(c["longest"], 1), device="cuda")
    x = torch.rand(c["batch"], c["kv_heads"], i.numel(), generator=g, device="cuda")
    x = torch.where((i < c["first"]) | (i >= (n - c["last"])[:, None, None]), 2.0, x)
    x = torch.where(i < n[:, None, None], x, -1.0).argsort(-1, descending=True)[..., :c["budget"]]
    j = torch.arange(x.shape[-1], device="cuda")
    x = torch.where(j < m[:, None, None], x, i.numel()).sort(-1).values
    kept = torch.full((c["batch"], c["kv_heads"], c["budget"]), -1, dtype=torch.int32, device="cuda")
    kept[..., :x.shape[-1]] = torch.where((j < m[:, None, None]) & (m < n)[:, None, None], x, -1)
    free = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    free[:40] = ids[sum(held):]
    s = {"kept": kept, "lengths": _int(lens), "stay": _int(stay), "table": table, "free": free, "n_free": _int([40]), "page": c["page"],
         "weights": _accounts(c, n_pages, g), "n_free_out": _int([0]), "status": _int([0])}
    for name in ("k", "v"):
        _pool(c, n_pages, lambda shape: torch.randn(shape, generator=g, device="cuda"), name, s)
    s["sizes"] = dict(max_pages=table.shape[1], n_pages=n_pages)
    if c["kv"] == "mxfp4":                                    # rows of what stays, to be read back
        rows = torch.cat([b * table.shape[1] * c["page"] + torch.arange(k, device="cuda") for b, k in enumerate(stay)])
        s["slots"] = table.reshape(-1)[rows // c["page"]].long() * c["page"] + rows % c["page"]
        s["k_out"], s["v_out"] = (torch.zeros(rows.numel(), c["kv_heads"], D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        s["sizes"]["max_tokens"] = max(rows.numel(), 1)
    return s


def prepare(case, seed):
    c = _full(case)
    g = _generator(seed)
    s = {"append": _prepare_append, "attention": _prepare_attention, "weights": _prepare_attention, "keep": _prepare_keep,
         "evict": _prepare_evict}[c["op"]](c, g)
    s["op"] = c["op"]
    sizes, back = s.pop("sizes"), s.pop("back_sizes", None)
    if own:                                                   # the parameter block and the scratch memory that a program keeps
        from paper_2410_16179_amd import binding as mp
        unit = 2 if c["kv"] == "mxfp4" else 1                 # elements of an entry of the tensor
        for name in ("k", "v"):
            if name + "_pages" in s:
                sizes[name + "_strides"] = tuple(unit * x for x in s[name + "_pages"].stride()[:3])
        both = dict(batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], dtype=c["dtype"], kv_dtype=c["kv"], page_size=c["page"])
        s["params"] = mp.make_paged_params(**both, **sizes)
        if back is not None:
            s["back_params"] = mp.make_paged_params(**both, **{**sizes, **back})
        s["ws"] = mp.alloc_paged_workspace(s["params"])
    return s


# ---- the operators' plain forms ----------------------------------------------------------------------
def _plain_append(s):
    pages, page = s["k_pages"].shape[:2]
    p = torch.div(s["slots"], page, rounding_mode="floor").clamp(min=0)
    at = (s["slots"] - p * page).clamp(min=0)
    keep = (s["slots"] >= 0)[:, None, None]
    # (the rows without a slot write what the first row does, which has one)
    lead = torch.where(s["slots"] >= 0, torch.arange(p.numel(), device=p.device), 0)
    p, at = p[lead], at[lead]
    got = {}
    for name in ("k", "v"):
        rows, scales = _quantised(s[name + "_new"].float())
        s[name + "_pages"][p, at], s[name + "_block"][p, at] = rows[lead], scales[lead]
        x = _values(s[name + "_pages"][p, at], s[name + "_block"][p, at])
        got[name] = torch.where(keep, x.to(s[name + "_out"].dtype), s[name + "_out"])
    return got


def _rows(s):
    """For every (request, new token): its row, whether it is there, and its position."""
    lens = s["lengths"].long()
    if s["token_start"] is None:
        t0 = torch.arange(lens.numel() + 1, device=lens.device)
    else:
        t0 = s["token_start"].long()
    n = t0[1:] - t0[:-1]
    t = torch.arange(s["new"], device=lens.device)
    there = t < n[:, None]
    return torch.where(there, t0[:-1, None] + t, s["q"].shape[0]), there, (lens - n)[:, None] + t


def _scores(s):
    """Rows, the pages and places of the keys, and the logits [batch, heads, new, group, keys]: -inf where a key is not attended."""
    lens, heads = s["lengths"].long(), s["k_pages"].shape[2]
    row, there, pos = _rows(s)
    batch, tokens = row.shape[0], s["q"].shape[0]
    i = torch.arange(s["longest"], device=lens.device)
    at = s["table"][:, i // s["page"]].long().clamp(min=0)
    seen = there[..., None] & (i <= pos[..., None])
    if s["local"]:
        seen = seen & ((i < s["sink"]) | (i > pos[..., None] - s["local"]))
    q = s["q"].float()[row.clamp(max=tokens - 1)]             # [batch, new, q_heads, D]
    q = q.reshape(batch, s["new"], heads, -1, D).transpose(1, 2).reshape(batch, heads, -1, D)
    x = torch.matmul(q, _keys(s, "k", at, i).transpose(2, 3)).mul_(1.0 / math.sqrt(D))
    x = x.reshape(batch, heads, s["new"], -1, s["longest"])
    return row, at, i, x.masked_fill_(~seen[:, None, :, None], -math.inf)


def _keys(s, name, at, i):
    """[batch, heads, keys, D]"""
    place, block = i % s["page"], s[name + "_block"]
    x = s[name + "_pages"][at, place]
    x = x.float() if block is None else _values(x, block[at, place])
    x = x if s["k_scale"] is None else x * s["k_scale"][:, None]
    return torch.where((i < s["lengths"][:, None])[..., None, None], x, 0.0).transpose(1, 2).contiguous()


def _plain_attention(s):
    row, at, i, x = _scores(s)
    batch, heads, tokens, q_heads = row.shape[0], s["k_pages"].shape[2], s["q"].shape[0], s["q"].shape[1]
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(batch, heads, -1, s["longest"]), _keys(s, "v", at, i))
    o = o.reshape(batch, heads, s["new"], -1, D)
    o = torch.where(total > 0, o / total, 0.0)
    out = torch.zeros(tokens + 1, q_heads, D, dtype=s["q"].dtype, device=o.device)
    lse = torch.zeros(tokens + 1, q_heads, device=o.device)
    out[row] = o.transpose(1, 2).reshape(batch, s["new"], q_heads, D).to(out.dtype)
    lse[row] = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(batch, s["new"], q_heads)
    return {"out": out[:tokens], "lse": lse[:tokens]}


def _plain_weights(s):
    row, at, i, x = _scores(s)
    batch, heads, tokens = row.shape[0], s["k_pages"].shape[2], s["q"].shape[0]
    lse = s["lse"][row.clamp(max=tokens - 1)].reshape(batch, s["new"], heads, -1).transpose(1, 2)
    lse = torch.where(lse == -math.inf, math.inf, lse)        # (a row that attends nothing adds nothing)
    add = x.sub_(lse[..., None]).exp_().sum((2, 3)).transpose(1, 2)             # [batch, keys, heads]
    lens, w, place = s["lengths"].long(), s["weights"], i % s["page"]
    old = torch.where((i < _rows(s)[2][:, :1])[..., None], w[at, :, place], 0.0)
    # (keys that are not there write to a page behind the last one)
    more = torch.cat([w, w[:1]])
    more[torch.where(i < lens[:, None], at, w.shape[0]), :, place] = old + add
    w.copy_(more[:w.shape[0]])
    return {"weights": w}


def _plain_keep(s):
    lens, most = s["lengths"].long(), s["kept"].shape[-1]
    i = torch.arange(s["longest"], device=lens.device)
    w = s["weights"][s["table"][:, i // s["page"]].long().clamp(min=0), :, i % s["page"]].transpose(1, 2)      # [batch, heads, keys]
    n = lens[:, None, None]
    w = torch.where((i < s["first"]) | (i >= n - s["last"]), math.inf, w)
    w = torch.where(i < n, w, -math.inf)
    stay = torch.minimum(lens, s["budgets"].long())
    goes = (stay < lens)[:, None, None]
    order = w.sort(dim=-1, descending=True, stable=True).indices[..., :most]
    j = torch.arange(order.shape[-1], device=lens.device)
    real = (j < stay[:, None, None]) & goes
    order = torch.where(real, order, s["longest"]).sort(-1).values
    kept = torch.full_like(s["kept"], -1)
    kept[..., :order.shape[-1]] = torch.where(real, order, -1)
    return {"kept": kept, "lengths": stay.to(torch.int32)}


def _plain_evict(s):
    batch, heads, most = s["kept"].shape
    page, table, lens, stay = s["page"], s["table"], s["lengths"].long(), s["stay"].long()
    j = torch.arange(min(most, table.shape[1] * page), device=lens.device)
    kept = s["kept"][..., :j.numel()].long()
    kept = torch.where(kept < 0, j, kept).clamp(max=table.shape[1] * page - 1)
    b = torch.arange(batch, device=lens.device)[:, None, None]
    h = torch.arange(heads, device=lens.device)[None, :, None]
    there = j < stay[:, None, None]
    spare = torch.zeros_like(j)
    src = table[b, torch.div(kept, page, rounding_mode="floor")].long().clamp(min=0)
    dst = table[:, torch.div(j, page, rounding_mode="floor")].long()[:, None].expand(src.shape)
    got = {}
    for name in ("k_pages", "v_pages", "k_block", "v_block", "weights"):
        pool = s[name]
        if pool is None:
            continue
        if pool.dtype == torch.float8_e4m3fn:
            pool = pool.view(torch.uint8)
        if name == "weights":
            pool = pool.transpose(1, 2)
        # (rows that are none go to a page behind the last one)
        more = torch.cat([pool, pool[:1]])
        more[torch.where(there, dst, pool.shape[0]), j % page + spare, h] = pool[src, kept % page, h]
        pool.copy_(more[:pool.shape[0]])
    held, left = (lens + page - 1) // page, (stay + page - 1) // page
    back = held - left
    r0 = back.cumsum(0)
    n_free = s["n_free"].long()
    x = torch.arange(s["free"].numel(), device=lens.device)
    r = (x - n_free).clamp(min=0)
    of = torch.searchsorted(r0, r, right=True).clamp(max=batch - 1)
    id_ = table[of, (left[of] + r - (r0[of] - back[of])).clamp(max=table.shape[1] - 1)]
    s["free"].copy_(torch.where((x >= n_free) & (r < r0[-1]), id_, s["free"]))
    got.update(weights=s["weights"], free=s["free"], n_free=(n_free + r0[-1]).to(torch.int32), status=torch.zeros_like(s["status"]))
    if s["k_block"] is None:
        return {**got, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    p, at = torch.div(s["slots"], page, rounding_mode="floor"), s["slots"] % page
    for name in ("k", "v"):
        got[name] = _values(s[name + "_pages"][p, at], s[name + "_block"][p, at]).to(torch.bfloat16)
    return got


# ---- the calls ---------------------------------------------------------------------------------------
def run(s):
    if not own:
        return {"append": _plain_append, "attention": _plain_attention, "weights": _plain_weights, "keep": _plain_keep,
                "evict": _plain_evict}[s["op"]](s)
    from paper_2410_16179_amd import binding as mp
    if s["op"] == "append":
        mp.magicpig_page_append_mxfp(s["params"], s["k_new"], s["v_new"], s["slots"], s["k_pages"], s["v_pages"], s["k_block"], s["v_block"])
        mp.magicpig_page_read_mxfp(s["back_params"], s["k_pages"], s["v_pages"], s["k_block"], s["v_block"], s["slots"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if s["op"] == "attention":
        mp.magicpig_paged_attention_mxfp(s["params"], s["q"], s["k_pages"], s["v_pages"], s["k_block"], s["v_block"], s["table"],
                                          s["lengths"], s["token_start"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if s["op"] == "weights":
        mp.magicpig_page_weights(s["params"], s["q"], s["k_pages"], s["k_scale"], s["k_block"], s["table"], s["lengths"],
                                 s["token_start"], s["lse"], None, s["weights"], s["ws"])
        return {"weights": s["weights"]}
    if s["op"] == "keep":
        mp.magicpig_page_keep(s["params"], s["weights"], s["table"], s["lengths"], s["budgets"], s["first"], s["last"], s["kept"],
                              s["lengths_out"], s["ws"])
        return {"kept": s["kept"], "lengths": s["lengths_out"]}
    mp.magicpig_page_evict(s["params"], s["kept"], s["lengths"], s["stay"], s["table"], s["free"], s["n_free"], s["k_pages"], s["v_pages"],
                           s["k_block"], s["v_block"], s["weights"], s["n_free_out"], s["status"], s["ws"])
    got = {"weights": s["weights"], "free": s["free"], "n_free": s["n_free_out"], "status": s["status"]}
    if s["k_block"] is None:
        return {**got, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    mp.magicpig_page_read_mxfp(s["params"], s["k_pages"], s["v_pages"], s["k_block"], s["v_block"], s["slots"], s["k_out"], s["v_out"])
    return {**got, "k": s["k_out"], "v": s["v_out"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------
_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_values(rows, scales):
    grid = torch.tensor(_GRID, dtype=torch.float64, device=rows.device)
    both = torch.stack([rows % 16, rows // 16], -1).flatten(-2).long()
    x = grid[both % 8] * (1 - 2 * (both // 8))
    return x * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _exact_rounded(x):
    """x [..., 128] in float64 to the nearest values of its blocks; of two as near the one with the even code."""
    top = x.unflatten(-1, (4, 32)).abs().amax(-1)
    power = torch.exp2(torch.ceil(torch.log2((top / 6.0).clamp(min=2.0 ** -127)) - 1e-12)).repeat_interleave(32, -1)
    y, got, best = x.abs() / power, torch.zeros_like(x), torch.full_like(x, math.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):
        off = (y - _GRID[code]).abs()
        got, best = torch.where(off < best, _GRID[code], got), torch.minimum(off, best)
    return got * power * torch.sign(x)


def _exact_key(s, c, name, pages, h, n):
    x = s[name + "_pages"][pages][:, :, h].flatten(0, 1)[:n]
    if s[name + "_block"] is not None:
        return _exact_values(x, s[name + "_block"][pages][:, :, h].flatten(0, 1)[:n])
    return x.double() if s["k_scale"] is None else x.double() * s["k_scale"][h].double()


def exact(case, seed):
    c = _full(case)
    if c["op"] == "keep":
        return None
    s = prepare(case, seed)
    if c["op"] == "append":
        got = {}
        for name in ("k", "v"):
            x = _exact_rounded(s[name + "_new"].double())
            got[name] = torch.where((s["slots"] >= 0)[:, None, None], x, 0.0)
        return got
    if c["op"] == "evict":
        four = c["kv"] == "mxfp4"
        pools = {name: s[name].double() for name in ("k_pages", "v_pages", "weights")} if not four else \
            {"k": _exact_values(s["k_pages"], s["k_block"]), "v": _exact_values(s["v_pages"], s["v_block"]), "weights": s["weights"].double()}
        for b, (n, m) in enumerate(zip(_lengths(c), _stay(c))):
            if m == n:
                continue
            for h in range(c["kv_heads"]):
                i, j = s["kept"][b, h, :m].long(), torch.arange(m, device="cuda")
                src, dst = s["table"][b, i // c["page"]].long(), s["table"][b, j // c["page"]].long()
                for name, x in pools.items():
                    if name == "weights":
                        x[dst, h, j % c["page"]] = x[src, h, i % c["page"]].clone()
                    else:
                        x[dst, j % c["page"], h] = x[src, i % c["page"], h].clone()
        got = {**pools, "free": None, "n_free": None, "status": None}
        if four:
            for name in ("k", "v"):
                got[name] = got[name][s["slots"] // c["page"], s["slots"] % c["page"]]
        return got
    G = c["q_heads"] // c["kv_heads"]
    if c["op"] == "weights":
        got = s["weights"].double()
    else:
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    row = 0
    for b, (n, t) in enumerate(zip(_lengths(c), _news(c))):
        pages = s["table"][b, :_up(n, c["page"])].long()
        p = torch.arange(n - t, n, device="cuda")[:, None]
        i = torch.arange(n, device="cuda")[None]
        hidden = i > p
        if c["local"]:
            hidden = hidden | ((i >= c["sink"]) & (i <= p - c["local"]))
        for h in range(c["kv_heads"]):
            if t == 0 or n == 0:
                if c["op"] == "attention":
                    lse[row:row + t, h * G:(h + 1) * G] = -math.inf
                continue
            K = _exact_key(s, c, "k", pages, h, n)
            V = _exact_key(s, c, "v", pages, h, n) if c["op"] == "attention" else None
            total = torch.zeros(n, dtype=torch.float64, device="cuda")
            for j in range(h * G, (h + 1) * G):
                x = s["q"][row:row + t, j].double() @ K.T / math.sqrt(D)
                x.masked_fill_(hidden, -math.inf)
                if V is None:
                    total += torch.exp(x - s["lse"][row:row + t, j, None].double()).sum(0)
                else:
                    lse[row:row + t, j] = torch.logsumexp(x, 1)
                    out[row:row + t, j] = torch.softmax(x, 1) @ V
            if V is None:
                at = s["table"][b, i[0] // c["page"]].long(), i[0] % c["page"]
                total[:n - t] += got[at[0][:n - t], h, at[1][:n - t]]
                got[at[0], h, at[1]] = total
        row += t
    return {"weights": got} if c["op"] == "weights" else {"out": out, "lse": lse}
