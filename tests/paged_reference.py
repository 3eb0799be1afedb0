"""Plain models of the paged cache's operators, in Python integers and 64-bit floats on the CPU, and the
tolerances that the kernels' arithmetic allows."""
from __future__ import annotations

import math

import numpy as np

D = 128


def plan(new, lengths, table, free, n_free, page, max_new, max_tokens):
    """What magicpig_page_plan leaves: a dict of numpy arrays (table and free are copies)."""
    batch, max_pages = table.shape
    table, free = table.copy(), free.copy()
    up = lambda n: -(-n // page)
    refused = {"lengths": np.array(lengths, np.int32), "n_free": n_free, "table": table, "free": free,
               "token_start": np.zeros(batch + 1, np.int32), "slots": np.full(max_tokens, -1, np.int64)}
    total, back, need = sum(max(n, 0) for n in new), [], 0
    wrong = total > max_tokens or n_free < 0
    for b in range(batch):
        n, held = int(new[b]), int(lengths[b])
        wrong |= n < -1 or n > max_new or held < 0 or held + max(n, 0) > max_pages * page
    if not wrong:
        back = [int(table[b, j]) for b in range(batch) if new[b] < 0 for j in range(up(int(lengths[b])))]
        need = sum(up(int(lengths[b] + new[b])) - up(int(lengths[b])) for b in range(batch) if new[b] >= 0)
        wrong = n_free + len(back) > len(free)
    if wrong:
        return {**refused, "status": -1}
    if need > n_free + len(back):
        return {**refused, "status": need - n_free - len(back)}
    stack = [int(x) for x in free[:n_free]] + back
    start, slots = [0], []
    out = np.zeros(batch, np.int32)
    for b in range(batch):
        if new[b] < 0:
            start.append(start[-1])
            continue
        for pos in range(int(lengths[b]), int(lengths[b] + new[b])):
            if pos % page == 0:
                table[b, pos // page] = stack.pop()
            slots.append(int(table[b, pos // page]) * page + pos % page)
        out[b] = lengths[b] + new[b]
        start.append(len(slots))
    free[n_free:len(stack)] = stack[n_free:]
    return {"lengths": out, "n_free": len(stack), "table": table, "free": free, "token_start": np.array(start, np.int32),
            "slots": np.array(slots + [-1] * (max_tokens - len(slots)), np.int64), "status": 0}


def attention(q, k_pages, v_pages, table, lengths, token_start, n_sink=0, n_local=0, scale=None, max_new=None):
    """q [tokens, heads, D], pools [pages, page, kv heads, D], all float64.  Returns out, lse, and for every row
    what the tolerances need: the attended |v| in the weights' mean, the largest sum of |q_d k_d|, and the
    number of keys; rows of no request are NaN."""
    tokens, heads, _ = q.shape
    pages, page, kv_heads, _ = k_pages.shape
    group = heads // kv_heads
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, size = np.full(q.shape, np.nan), np.zeros(q.shape)
    lse, reach, count = np.full((tokens, heads), np.nan), np.zeros((tokens, heads)), np.zeros((tokens, heads))
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for b, n in enumerate(lengths):
            n = int(n)
            first, last = (b, b + 1) if token_start is None else (int(token_start[b]), int(token_start[b + 1]))
            new = last - first if max_new is None else min(last - first, max_new)
            i = np.arange(n)
            ids = table[b, i // page]
            held = (ids >= 0) & (ids < pages)
            for t in range(new):
                p = n - (last - first if max_new is None else new) + t
                seen = held & (i <= p)
                if n_local:
                    seen &= (i < n_sink) | (i > p - n_local)
                at = np.nonzero(seen)[0]
                for h in range(heads):
                    g, r = h // group, first + t
                    if len(at) == 0:
                        out[r, h], lse[r, h] = 0.0, -np.inf
                        continue
                    K, V = k_pages[ids[at], at % page, g], v_pages[ids[at], at % page, g]
                    x = K @ q[r, h] * scale
                    top = x.max()
                    w = np.exp(x - top)
                    out[r, h] = w @ V / w.sum()
                    lse[r, h] = top + np.log(w.sum())
                    size[r, h] = w @ np.abs(V) / w.sum()
                    reach[r, h] = (np.abs(K) @ np.abs(q[r, h])).max() * abs(scale)
                    count[r, h] = len(at)
    return out, lse, size, reach, count


def tolerance(out, size, reach, count, dtype, rounded_weights):
    """How far an output may be off.  A score is a float32 sum of 128 products (each addition off by at most
    2^-24 of the running magnitude, some more for the scalings): 132 * 2^-24 * sum |q k|; it moves a weight, and the sum
    of the weights, by as much relatively.  The weighted sum and the sum of the weights are float32 sums over the
    keys (2^-23 per key, both together; 64 more for exponentials, rescaling and joining).  bf16: the weights are taken to
    2^-16 (two bf16), or to half a step of bf16 where a wavefront takes many rows; the output is rounded once, by
    half a step at most."""
    part = 2 * 132 * 2.0 ** -24 * reach + (count + 64) * 2.0 ** -23
    if dtype != "fp32":
        part = part + (2.0 ** -8 if rounded_weights else 2.0 ** -16)
    last = 2.0 ** -24 if dtype == "fp32" else 2.0 ** -8
    return size * part[..., None] + last * np.abs(out) * (1 + part[..., None]) + 1e-37


def lse_tolerance(lse, reach, count):
    return 132 * 2.0 ** -24 * reach + (count + 64) * 2.0 ** -23 + 4 * 2.0 ** -24 * np.abs(np.where(np.isfinite(lse), lse, 0))
