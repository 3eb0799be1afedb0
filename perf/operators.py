"""The paged key-value cache and the exact attention that reads it, as cases that can be timed and checked.

A serving program keeps the keys and values of all its requests in one pool of pages per layer.  Three
operators deal with it:

  plan       requests' lengths and new tokens -> pages handed out and taken back, block tables, slot maps
  append     the new tokens' keys and values go to their slots of the pool
  attention  the new tokens attend their requests' cached keys, through the block tables: one token per
             request (decoding), a few (verification of drafted tokens), or a prompt or a chunk of one

`own` selects between the operators' plain forms (elementary torch operations in float32) and the calls of
this library.  Both take what prepare() gives.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "fp8": 1}

_DEFAULT = {"batch": 1, "q_heads": 32, "kv_heads": 8, "dtype": "bf16", "kv": "", "page": 64, "shortest": 0, "longest": 0,
            "new": 1, "fewest": 0, "sink": 0, "local": 0, "layout": "token", "tokens": 0, "mix": False}


def _case(name, op, **more):
    c = {"name": name, "op": op}
    c.update({k: v for k, v in more.items() if _DEFAULT[k] != v})
    return c


def _full(case):
    return {**_DEFAULT, **case}


def listed():
    return [
        # the bookkeeping of a decoding step: every request gets one token, one in `page` of them a page
        _case("plan_decode_b64", "plan", batch=64, shortest=500, longest=60000),
        # a large engine's step: decoding requests, prompts of up to 2048 tokens, requests that end and idle places
        _case("plan_mixed_b512", "plan", batch=512, page=16, shortest=1, longest=8192, new=2048, mix=True),
        # the new token of each of 64 requests
        _case("append_b64", "append", tokens=64),
        # a step full of prompt tokens, into a quantised pool stored head by head, with a scale per head
        _case("append_16k_fp8", "append", tokens=16384, kv="fp8", page=32, layout="head"),
        # a short conversation of one user: nothing but latency and launches
        _case("decode_2k", "attention", page=16, shortest=2048, longest=2048),
        # one user at 96k tokens (the shape of C3)
        _case("decode_96k", "attention", shortest=98304, longest=98304),
        # a serving batch of 64k contexts (the shape of C4)
        _case("decode_b16_64k", "attention", batch=16, shortest=65536, longest=65536, page=128, layout="head"),
        # a ragged batch, eight query heads per KV head, quantised pool
        _case("decode_ragged_fp8", "attention", batch=48, q_heads=64, page=32, kv="fp8", shortest=50, longest=30011),
        # float32 from end to end, every head with keys of its own
        _case("decode_fp32_mha", "attention", batch=6, q_heads=32, kv_heads=32, dtype="fp32", shortest=333, longest=9001),
        # up to four drafted tokens a request are verified, five heads per KV head; sink tokens and a local window
        _case("verify_window", "attention", batch=24, q_heads=40, page=16, shortest=700, longest=20000, new=4, fewest=1,
              sink=4, local=4096),
        # prompts from nothing, one long and three shorter ones
        _case("prompt_b4", "attention", batch=4, shortest=1000, longest=4099, new=4099, fewest=4099),
        # a chunk of a long prompt behind what is cached of it already
        _case("chunk_60k", "attention", shortest=61440, longest=61440, new=2048, fewest=2048),
    ]


# (query heads, KV heads)
_HEADS = [(32, 8), (32, 8), (64, 8), (40, 8), (28, 4), (16, 2), (8, 1), (24, 8), (8, 8), (32, 32), (1, 1)]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attention", "attention", "attention", "attention"])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256])
    hq, hkv = rng.choice(_HEADS)
    dtype, kv = rng.choice([("bf16", ""), ("bf16", ""), ("bf16", "fp8"), ("fp32", "")])
    layout = rng.choice(["token", "head"])
    if op == "plan":
        mix = rng.random() < 0.6
        longest = _between(rng, 64, 60000)
        got = _case("", op, batch=_between(rng, 1, 1500), page=page, shortest=rng.randint(0, longest), longest=longest,
                    new=_between(rng, 2, 2048) if mix else 1, mix=mix)
    elif op == "append":
        got = _case("", op, tokens=_between(rng, 1, 16384), q_heads=hq, kv_heads=hkv, dtype=dtype, kv=kv, page=page, layout=layout)
    else:
        kind = rng.choice(["decode", "decode", "verify", "prompt"])
        longest = _between(rng, 1, 100000)
        shortest = rng.choice([longest, rng.randint(0, longest), rng.randint(0, longest)])
        new, fewest = {"decode": (1, 1), "verify": (rng.randint(2, 8), 1), "prompt": (_between(rng, 16, 4096),) * 2}[kind]
        new = min(new, longest)
        local = rng.choice([0, 0, 0, _between(rng, 16, 8192)])
        c = dict(q_heads=hq, kv_heads=hkv, dtype=dtype, kv=kv, page=page, layout=layout, shortest=shortest, longest=longest,
                 new=new, fewest=min(fewest, new), sink=rng.choice([0, 4, 20]) if local else 0, local=local)
        c["batch"] = _between(rng, 1, 128)
        # no more keys, scores and work than the largest listed cases
        while c["batch"] > 1 and _too_much({**c, "op": op}):
            c["batch"] = c["batch"] * 2 // 3
        while _too_much({**c, "op": op}):
            c["new"] = c["new"] * 2 // 3
            c["fewest"] = min(c["fewest"], c["new"])
        got = _case("", op, **c)
    del got["name"]
    return got


def _too_much(case):
    c = _full(case)
    rows = c["batch"] * c["new"] * c["q_heads"]
    return (c["batch"] * c["longest"] * c["kv_heads"] * D * _BYTES[c["kv"] or c["dtype"]] > 2.2e9 or rows * c["longest"] > 4.2e9
            or c["batch"] * c["longest"] * c["kv_heads"] * D > 1.1e9 or work(c)["flops"] > (2e12 if c["dtype"] == "bf16" else 4e11))


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
    """attention: the new tokens of the requests (among the lengths).  plan: behind the lengths; -1: the request ends."""
    if c["op"] == "plan":
        if not c["mix"]:
            return [1] * c["batch"]
        kinds, sizes = _spread(c["batch"], 1), _spread(c["batch"], 2)
        return [1 if k < 0.8 else -1 if k < 0.86 else 0 if k < 0.9 else max(1, int(c["new"] * s)) for k, s in zip(kinds, sizes)]
    if c["new"] == 1:
        return [1] * c["batch"]                               # (also where nothing is cached: a row that attends no key)
    if c["fewest"] == c["new"]:
        return [min(n, c["new"]) for n in _lengths(c)]
    return [min(n, max(1, c["fewest"] + int((c["new"] - c["fewest"] + 1) * f))) for n, f in zip(_lengths(c), _spread(c["batch"], 1))]


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
    if c["op"] == "plan":
        lens, news = _lengths(c), _news(c)
        tokens = _tokens(c)
        opened = sum(_up(n + t, c["page"]) - _up(n, c["page"]) for n, t in zip(lens, news) if t > 0)
        closed = sum(_up(n, c["page"]) for n, t in zip(lens, news) if t < 0)
        # lengths and new tokens in, lengths and starts out; a slot for every token; an id read and written for every page
        return {"bytes": 16 * c["batch"] + 8 * tokens + 8 * (opened + closed) + 16, "flops": 0}
    row = c["kv_heads"] * D
    if c["op"] == "append":
        return {"bytes": c["tokens"] * (2 * row * (_BYTES[c["dtype"]] + _BYTES[c["kv"] or c["dtype"]]) + 8), "flops": 0}
    pairs, read, tokens = 0, 0, 0
    for n, t in zip(_lengths(c), _news(c)):
        a, k = _attended(c, n, t)
        pairs, read, tokens = pairs + a, read + k, tokens + t
    return {"bytes": read * 2 * row * _BYTES[c["kv"] or c["dtype"]] + tokens * c["q_heads"] * (2 * D * _BYTES[c["dtype"]] + 4),
            "flops": 4 * D * c["q_heads"] * pairs}


# ---- inputs ------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 31) + 29)
    return g


def _store(x, kind):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn) if kind == "fp8" else x.to(_TYPES[kind])


def _pool(c, pages, fill):
    """[pages, page, kv heads, D], a view in the case's layout; fill(shape) gives float32 values (in parts: they are larger)."""
    shape = (pages, c["kv_heads"], c["page"], D) if c["layout"] == "head" else (pages, c["page"], c["kv_heads"], D)
    t = torch.zeros(shape, dtype=_TYPES[c["kv"] or c["dtype"]], device="cuda")
    if fill is not None:
        part = max(1, (1 << 27) // (c["page"] * c["kv_heads"] * D))
        for a in range(0, pages, part):
            b = min(pages, a + part)
            t[a:b] = _store(fill((b - a,) + shape[1:]), c["kv"] or c["dtype"])
    return t.permute(0, 2, 1, 3) if c["layout"] == "head" else t


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _scales(c, g):
    if c["kv"] != "fp8":
        return None, None
    return tuple(0.01 + 0.02 * torch.rand(c["kv_heads"], generator=g, device="cuda") for _ in range(2))


def _tokens(c):
    """Rows of the token arrays of a plan: the step's tokens, rounded up as an engine's buffers are."""
    return _up(sum(max(0, t) for t in _news(c)), 64) * 64


def _prepare_plan(c, g):
    lens, news = _lengths(c), _news(c)
    held = [_up(n, c["page"]) for n in lens]
    opened = sum(_up(n + t, c["page"]) - h for n, t, h in zip(lens, news, held) if t > 0)
    max_pages = max(_up(n + max(t, 0), c["page"]) for n, t in zip(lens, news)) + 1
    n_pages = sum(held) + opened + 64
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    at = torch.arange(max_pages, device="cuda")
    count = torch.tensor(held, device="cuda")
    first = count.cumsum(0) - count
    table = torch.where(at < count[:, None], ids[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    free = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    n_free = n_pages - sum(held)
    free[:n_free] = ids[sum(held):]
    s = {"new": _int(news), "lengths": _int(lens), "table": table, "free": free, "n_free": _int([n_free]), "page": c["page"],
         "token_start": torch.zeros(c["batch"] + 1, dtype=torch.int32, device="cuda"),
         "slots": torch.zeros(_tokens(c), dtype=torch.int64, device="cuda"), "status": _int([0]),
         "lengths_out": torch.zeros(c["batch"], dtype=torch.int32, device="cuda"), "n_free_out": _int([0]),
         "max_new": max(max(news), 1)}
    s["sizes"] = dict(max_pages=max_pages, n_pages=n_pages, max_tokens=_tokens(c), max_new=s["max_new"])
    return s


def _prepare_append(c, g):
    n = c["tokens"]
    pages = _up(n, c["page"]) + 3
    wide = c["q_heads"] + 2 * c["kv_heads"]                  # the projections of a layer come from one product
    qkv = torch.randn(n, wide, D, generator=g, device="cuda").to(_TYPES[c["dtype"]])
    i = torch.arange(n, device="cuda")
    ids = torch.randperm(pages, generator=g, device="cuda")
    slots = ids[i // c["page"]] * c["page"] + i % c["page"]
    slots = torch.where(i < n - n // 16, slots, -1)           # (rows behind the step's tokens)
    k_scale, v_scale = _scales(c, g)
    s = {"k_new": qkv[:, c["q_heads"]:c["q_heads"] + c["kv_heads"]], "v_new": qkv[:, c["q_heads"] + c["kv_heads"]:], "slots": slots,
         "k_scale": k_scale, "v_scale": v_scale, "k_pages": _pool(c, pages, None), "v_pages": _pool(c, pages, None)}
    s["sizes"] = dict(max_pages=pages, n_pages=pages, max_tokens=n, max_new=n, k_new_strides=s["k_new"].stride()[:2],
                      v_new_strides=s["v_new"].stride()[:2])
    return s


def _prepare_attention(c, g):
    lens, news = _lengths(c), _news(c)
    held = [_up(n, c["page"]) for n in lens]
    max_pages, n_pages, tokens = max(max(held), 1), sum(held) + 2, sum(news) + (3 if c["new"] > 1 else 0)
    count = torch.tensor(held, device="cuda")
    first = count.cumsum(0) - count
    at = torch.arange(max_pages, device="cuda")
    ids = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.where(at < count[:, None], ids[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    k_scale, v_scale = _scales(c, g)
    k_size, v_size = (1.0, 1.0) if k_scale is None else (50.0, 50.0)
    # keys of a head share an offset, as cached keys do; queries that make a few keys stand out
    shift = torch.randn(c["kv_heads"], 1, D, generator=g, device="cuda") if c["layout"] == "head" else \
        torch.randn(c["kv_heads"], D, generator=g, device="cuda")
    k_pages = _pool(c, n_pages, lambda shape: k_size * (torch.randn(shape, generator=g, device="cuda") + shift))
    v_pages = _pool(c, n_pages, lambda shape: v_size * (0.3 + torch.randn(shape, generator=g, device="cuda")))
    q = (1.5 * torch.randn(tokens, c["q_heads"], D, generator=g, device="cuda")).to(_TYPES[c["dtype"]])
    start = [sum(news[:b]) for b in range(c["batch"] + 1)]
    s = {"q": q, "k_pages": k_pages, "v_pages": v_pages, "k_scale": k_scale, "v_scale": v_scale, "table": table,
         "lengths": _int(lens), "token_start": _int(start) if c["new"] > 1 else None, "page": c["page"], "new": c["new"],
         "longest": max(c["longest"], 1), "sink": c["sink"], "local": c["local"],
         "out": torch.zeros_like(q), "lse": torch.zeros(tokens, c["q_heads"], device="cuda")}
    s["sizes"] = dict(max_pages=max_pages, n_pages=n_pages, max_tokens=tokens, max_new=c["new"], n_sink=c["sink"], n_local=c["local"])
    return s


def prepare(case, seed):
    c = _full(case)
    g = _generator(seed)
    s = {"plan": _prepare_plan, "append": _prepare_append, "attention": _prepare_attention}[c["op"]](c, g)
    s["op"] = c["op"]
    sizes = s.pop("sizes")
    if own:                                                   # the parameter block and the scratch memory that a program keeps
        from paper_2410_16179_amd import binding as mp
        pools = {} if c["op"] == "plan" else {"k_strides": s["k_pages"].stride()[:3], "v_strides": s["v_pages"].stride()[:3]}
        s["params"] = mp.make_paged_params(batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], dtype=c["dtype"],
                                           kv_dtype=c["kv"], page_size=c["page"], **sizes, **pools)
        s["ws"] = mp.alloc_paged_workspace(s["params"])
    return s


# ---- the operators' plain forms ----------------------------------------------------------------------
def _plain_plan(s):
    new, lens, table, free, page = (s[k] for k in ("new", "lengths", "table", "free", "page"))
    batch, max_pages = table.shape
    new, lens, n_free = new.long(), lens.long(), s["n_free"].long()
    ended, n = new < 0, new.clamp(min=0)
    held = (lens + page - 1) // page
    need = torch.where(ended, 0, (lens + n + page - 1) // page - held)
    back = torch.where(ended, held, 0)
    zero = torch.zeros(1, dtype=torch.int64, device=new.device)
    t0, a0, r0 = (torch.cat([zero, x.cumsum(0)]) for x in (n, need, back))
    wrong = ((new < -1) | (new > s["max_new"]) | (lens < 0) | (lens + n > max_pages * page)).any()
    wrong = wrong | (t0[-1] > s["slots"].numel()) | (n_free < 0) | (n_free + r0[-1] > free.numel())
    status = torch.where(wrong, -1, (a0[-1:] - n_free - r0[-1:]).clamp(min=0)).to(torch.int32)
    fine = status == 0

    def stacked(x):                                           # entry x of the free stack with the ended requests' pages on top
        r = (x - n_free).clamp(min=0)
        b = (torch.searchsorted(r0, r, right=True) - 1).clamp(0, batch - 1)
        return torch.where(x < n_free, free[x.clamp(0, free.numel() - 1)], table[b, (r - r0[b]).clamp(0, max_pages - 1)])

    i = torch.arange(s["slots"].numel(), device=new.device)
    b = (torch.searchsorted(t0, i, right=True) - 1).clamp(0, batch - 1)
    pos = lens[b] + i - t0[b]
    p = pos // page
    opened = p >= held[b]
    ids = torch.where(opened, stacked(n_free + r0[-1] - 1 - (a0[b] + p - held[b])), table[b, p.clamp(max=max_pages - 1)]).long()
    real = (i < t0[-1]) & fine
    slots = torch.where(real, ids * page + pos % page, -1)
    spare = batch * max_pages
    at = torch.where(real & opened & (pos % page == 0), b * max_pages + p, spare)
    flat = torch.cat([table.reshape(-1), table.new_zeros(1)]).scatter(0, at, ids.to(torch.int32))[:spare]
    x = torch.arange(free.numel(), device=new.device)
    kept = (x >= n_free) & (x < n_free + r0[-1] - a0[-1]) & fine
    return {"lengths": torch.where(fine, torch.where(ended, 0, lens + n), lens).to(torch.int32), "table": flat.reshape(table.shape),
            "free": torch.where(kept, stacked(x), free), "n_free": torch.where(fine, n_free + r0[-1] - a0[-1], n_free).to(torch.int32),
            "token_start": torch.where(fine, t0, 0).to(torch.int32), "slots": slots, "status": status}


def _plain_append(s):
    pages, page = s["k_pages"].shape[:2]
    keep = s["slots"] >= 0
    slots = torch.where(keep, s["slots"], pages * page)

    def put(x, pool, scale):
        x = x.float()
        if scale is not None:
            x = x / scale[:, None]
        if pool.dtype == torch.float8_e4m3fn:
            x = x.clamp(-448.0, 448.0)
        p = torch.div(slots, page, rounding_mode="floor")
        as_bytes = torch.uint8 if pool.dtype == torch.float8_e4m3fn else pool.dtype
        rows = x.to(pool.dtype).view(as_bytes)
        # (a page behind the last one takes the rows that have no slot)
        more = torch.cat([pool.view(as_bytes), torch.zeros_like(pool[:1].view(as_bytes))])
        more[p, slots - p * page] = rows
        return more[:pages].view(pool.dtype)

    return {"k_pages": put(s["k_new"], s["k_pages"], s["k_scale"]), "v_pages": put(s["v_new"], s["v_pages"], s["v_scale"])}


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


def _plain_attention(s):
    lens, heads = s["lengths"].long(), s["k_pages"].shape[2]
    row, there, pos = _rows(s)
    batch, tokens, q_heads = row.shape[0], s["q"].shape[0], s["q"].shape[1]
    i = torch.arange(s["longest"], device=lens.device)
    at = s["table"][:, i // s["page"]].long().clamp(min=0)
    cached = (i < lens[:, None])[..., None, None]

    def keys(pool, scale):                                    # [batch, heads, keys, D]
        x = pool[at, i % s["page"]].float()
        x = x if scale is None else x * scale[:, None]
        return torch.where(cached, x, 0.0).transpose(1, 2).contiguous()

    seen = there[..., None] & (i <= pos[..., None])
    if s["local"]:
        seen = seen & ((i < s["sink"]) | (i > pos[..., None] - s["local"]))
    q = s["q"].float()[row.clamp(max=tokens - 1)]             # [batch, new, q_heads, D]
    q = q.reshape(batch, s["new"], heads, -1, D).transpose(1, 2).reshape(batch, heads, -1, D)
    x = torch.matmul(q, keys(s["k_pages"], s["k_scale"]).transpose(2, 3)).mul_(1.0 / math.sqrt(D))
    x = x.reshape(batch, heads, s["new"], -1, s["longest"])
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(batch, heads, -1, s["longest"]), keys(s["v_pages"], s["v_scale"]))
    o = o.reshape(batch, heads, s["new"], -1, D)
    o = torch.where(total > 0, o / total, 0.0)
    out = torch.zeros(tokens + 1, q_heads, D, dtype=s["q"].dtype, device=q.device)
    lse = torch.zeros(tokens + 1, q_heads, device=q.device)
    out[row] = o.transpose(1, 2).reshape(batch, s["new"], q_heads, D).to(out.dtype)
    lse[row] = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(batch, s["new"], q_heads)
    return {"out": out[:tokens], "lse": lse[:tokens]}


# ---- the calls ---------------------------------------------------------------------------------------
def run(s):
    if not own:
        return {"plan": _plain_plan, "append": _plain_append, "attention": _plain_attention}[s["op"]](s)
    from paper_2410_16179_amd import binding as mp
    if s["op"] == "plan":
        mp.magicpig_page_plan(s["params"], s["new"], s["lengths"], s["table"], s["free"], s["n_free"], s["lengths_out"],
                              s["n_free_out"], s["token_start"], s["slots"], s["status"], s["ws"])
        return {"lengths": s["lengths_out"], "table": s["table"], "free": s["free"], "n_free": s["n_free_out"],
                "token_start": s["token_start"], "slots": s["slots"], "status": s["status"]}
    if s["op"] == "append":
        mp.magicpig_page_append(s["params"], s["k_new"], s["v_new"], s["slots"], s["k_scale"], s["v_scale"], s["k_pages"],
                                s["v_pages"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    mp.magicpig_paged_attention(s["params"], s["q"], s["k_pages"], s["v_pages"], s["k_scale"], s["v_scale"], s["table"],
                                s["lengths"], s["token_start"], s["out"], s["lse"], s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------
def exact(case, seed):
    c = _full(case)
    if c["op"] == "plan":
        return None
    s = prepare(case, seed)
    if c["op"] == "append":
        got = {}
        for name in ("k", "v"):
            pool = s[name + "_pages"].double()
            new, scale = s[name + "_new"].double(), s[name + "_scale"]
            if scale is not None:
                new = (new / scale.double()[:, None]).clamp(-448.0, 448.0)
            for t, slot in enumerate(s["slots"].tolist()):
                if slot >= 0:
                    pool[slot // c["page"], slot % c["page"]] = new[t]
            got[name + "_pages"] = pool
        return got
    G = c["q_heads"] // c["kv_heads"]
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
            K = s["k_pages"][pages][:, :, h].reshape(-1, D)[:n].double()
            V = s["v_pages"][pages][:, :, h].reshape(-1, D)[:n].double()
            if c["kv"] == "fp8":
                K, V = K * s["k_scale"][h].double(), V * s["v_scale"][h].double()
            for j in range(h * G, (h + 1) * G):
                if t == 0 or n == 0:
                    lse[row:row + t, j] = -math.inf
                    continue
                x = s["q"][row:row + t, j].double() @ K.T / math.sqrt(D)
                x.masked_fill_(hidden, -math.inf)
                lse[row:row + t, j] = torch.logsumexp(x, 1)
                out[row:row + t, j] = torch.softmax(x, 1) @ V
        row += t
    return {"out": out, "lse": lse}
