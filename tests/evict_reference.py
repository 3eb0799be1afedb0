"""Plain models of the accounts of attention weight and of eviction, in 64-bit floats and Python integers on the CPU."""
from __future__ import annotations

import math

import numpy as np

D = 128


def weights(q, k_pages, table, lengths, token_start, lse, counted, accounts, n_sink=0, n_local=0, scale=None, max_new=None):
    """q [tokens, heads, D], k_pages [pages, page, kv heads, D], accounts [pages, kv heads, page], float64.  Returns the accounts and, for
    each, how far float32 may be off: a score is a float32 sum of 128 products (132 * 2^-24 * sum |q k| with its scaling), the
    difference to lse is rounded (2^-24 of either, twice for the change to base 2), the exponential is off by two units, and every
    addition by half a unit of what has been added up."""
    tokens, heads, _ = q.shape
    pages, page, kv_heads, _ = k_pages.shape
    group = heads // kv_heads
    scale = 1 / math.sqrt(D) if scale is None else scale
    got, off = accounts.copy(), np.zeros(accounts.shape)
    with np.errstate(invalid="ignore", over="ignore"):
        for b, n in enumerate(int(x) for x in lengths):
            first, last = (b, b + 1) if token_start is None else (int(token_start[b]), int(token_start[b + 1]))
            new = last - first if max_new is None else min(last - first, max_new)
            i = np.arange(n)
            ids = table[b, i // page]
            held = (ids >= 0) & (ids < pages)
            c = n - new if counted is None else int(counted[b])
            c = min(max(c, 0), n)
            for g in range(kv_heads):
                add, err, rows = np.zeros(n), np.zeros(n), 0
                at = np.nonzero(held)[0]
                K = np.zeros((n, D))
                K[at] = k_pages[ids[at], at % page, g]
                for t in range(new):
                    p = n - new + t
                    seen = held & (i <= p)
                    if n_local:
                        seen &= (i < n_sink) | (i > p - n_local)
                    for h in range(g * group, (g + 1) * group):
                        r = first + t
                        if lse[r, h] == -np.inf:
                            continue
                        x = K[seen] @ q[r, h] * scale
                        w = np.exp(x - lse[r, h])
                        reach = np.abs(K[seen]) @ np.abs(q[r, h]) * abs(scale)
                        add[seen] += w
                        err[seen] += w * (132 * 2.0 ** -24 * reach + 2.0 ** -22 * (np.abs(x) + abs(lse[r, h]) + 2))
                        rows += 1
                old = np.where(i < c, 0.0, 0.0)
                old[at] = np.where(at < c, accounts[ids[at], g, at % page], 0.0)
                total = old + add
                got[ids[at], g, at % page] = total[at]
                off[ids[at], g, at % page] = (err + (rows + 12) * 2.0 ** -24 * (np.abs(old) + add))[at]
    return got, off


def keep(accounts, table, lengths, budgets, n_first, n_last, max_keep):
    pages, kv_heads, page = accounts.shape
    batch = len(lengths)
    kept, out = np.full((batch, kv_heads, max_keep), -1, np.int32), np.array(lengths, np.int32)
    for b, n in enumerate(int(x) for x in lengths):
        budget = int(budgets[b])
        stay = n if budget < 0 else min(n, budget, max_keep)
        out[b] = stay
        if stay == n:
            continue
        i = np.arange(n)
        ids = table[b, i // page]
        held = (ids >= 0) & (ids < pages)
        for g in range(kv_heads):
            w = np.full(n, np.nan)
            w[held] = accounts[ids[held], g, i[held] % page]
            sure = (i < n_first) | (i >= n - n_last)
            # NaN below -inf; zeros alike
            order = sorted(range(n), key=lambda x: (not sure[x], np.isnan(w[x]), 0.0 if np.isnan(w[x]) or sure[x] else -w[x], x))
            kept[b, g, :stay] = sorted(order[:stay])
    return kept, out


def evict(kept, lengths, stay, table, free, n_free, page, arrays):
    """arrays: numpy arrays [pages, page, kv heads, ..], changed in place.  Returns free pages, their number and the status."""
    batch, max_pages = table.shape
    up = lambda n: -(-int(n) // page)
    for n, m in zip(lengths, stay):
        if n < 0 or n > max_pages * page or m < 0 or m > n or (kept is not None and m < n and m > kept.shape[-1]):
            return free, n_free, -1
    back = [int(table[b, j]) for b in range(batch) for j in range(up(stay[b]), up(lengths[b]))]
    if n_free < 0 or n_free + len(back) > len(free):
        return free, n_free, -1
    if kept is not None:
        for b in range(batch):
            if stay[b] == lengths[b]:
                continue
            for g in range(kept.shape[1]):
                for j in range(int(stay[b])):
                    i = int(kept[b, g, j])
                    if not j < i < lengths[b]:
                        continue
                    src, dst = int(table[b, i // page]), int(table[b, j // page])
                    for x in arrays:
                        x[dst, j % page, g] = x[src, i % page, g]
    free = free.copy()
    free[n_free:n_free + len(back)] = back
    return free, n_free + len(back), 0
