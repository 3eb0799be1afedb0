"""Which keys stay, exactly."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import evict_reference as ev

pytestmark = pytest.mark.gpu


def problem(rng, lengths, kv_heads, page, accounts=None):
    held = [-(-n // page) for n in lengths]
    max_pages, n_pages = max(max(held), 1) + 1, sum(held) + 2
    ids = rng.permutation(n_pages)[:sum(held)]
    table, at = np.full((len(lengths), max_pages), -1, np.int32), 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h]
        at += h
    shape = (n_pages, kv_heads, page)
    w = rng.standard_normal(shape) if accounts is None else accounts(rng, shape)
    return table, w.astype(np.float32)


def run(table, w, lengths, budgets, n_first, n_last, max_keep):
    pages, kv_heads, page = w.shape
    p = mp.make_paged_params(batch=len(lengths), n_q_heads=kv_heads, n_kv_heads=kv_heads, dtype="bf16", page_size=page, max_pages=table.shape[1],
                             n_pages=pages)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    kept = torch.full((len(lengths), kv_heads, max_keep), 12345, dtype=torch.int32, device="cuda")
    out = torch.full((len(lengths),), -9, dtype=torch.int32, device="cuda")
    mp.magicpig_page_keep(p, torch.from_numpy(w).cuda(), i32(table), i32(lengths), i32(budgets), n_first, n_last, kept, out, mp.alloc_paged_workspace(p))
    return kept.cpu().numpy(), out.cpu().numpy()


def check(seed, lengths, budgets, n_first=0, n_last=0, max_keep=None, kv_heads=2, page=16, accounts=None, bad=()):
    rng = np.random.default_rng(seed)
    table, w = problem(rng, lengths, kv_heads, page, accounts)
    for b, j, value in bad:
        table[b, j] = value
    max_keep = max(max(budgets), 1) if max_keep is None else max_keep
    kept, out = run(table, w, lengths, budgets, n_first, n_last, max_keep)
    want, want_out = ev.keep(w, table, lengths, budgets, n_first, n_last, max_keep)
    np.testing.assert_array_equal(out, want_out)
    np.testing.assert_array_equal(kept, want)


EDGES = [0, 1, 2, 15, 16, 17, 63, 64, 65, 300, 1023, 1024, 1025, 4095, 4096, 4097, 5000]


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("budget", [0, 1, 7, 64, 1000])
@pytest.mark.parametrize("n_first,n_last", [(0, 0), (4, 0), (0, 5), (4, 60), (900, 900)])
def test_budgets(page, budget, n_first, n_last):
    check(budget + page, EDGES, [budget] * len(EDGES), n_first, n_last, page=page)


@pytest.mark.parametrize("kv_heads", [1, 3, 8])
def test_budgets_of_their_own(kv_heads):
    # none, those that are not reached, larger ones than there is room for
    check(kv_heads, [100, 200, 300, 400, 500, 600], [-1, 0, 300, 399, 5000, -2 ** 31], max_keep=350, n_first=2, n_last=9, kv_heads=kv_heads)
    check(kv_heads, [700, 50], [2 ** 31 - 1, 49], max_keep=1, kv_heads=kv_heads)


@pytest.mark.parametrize("accounts", [
    lambda rng, s: np.zeros(s), lambda rng, s: rng.integers(0, 3, s) * 0.5, lambda rng, s: np.where(rng.random(s) < 0.5, 0.0, -0.0),
    lambda rng, s: np.exp(60 * rng.standard_normal(s)), lambda rng, s: -np.exp(3 * rng.standard_normal(s)),
    lambda rng, s: rng.integers(-3, 4, s) * 2.0 ** -149, lambda rng, s: 1 + rng.integers(0, 300, s) * 2.0 ** -23,
    lambda rng, s: rng.choice([np.nan, np.inf, -np.inf, 1.0, 2.0, -1.0], s), lambda rng, s: np.full(s, np.nan)])
def test_ties_and_values_of_every_kind(accounts):
    with np.errstate(over="ignore"):
        check(1, [5000, 900, 4096], [333, 899, 2000], 3, 10, accounts=accounts)
        check(2, [5000, 900, 4096], [333, 899, 2000], accounts=accounts)


def test_pages_that_are_none_come_last():
    check(3, [90, 64, 3000], [40, 60, 100], 1, 2, bad=[(0, 1, -1), (0, 3, 1 << 30), (1, 0, -2 ** 31), (2, 100, 10 ** 6)])
    check(4, [90], [89], bad=[(0, j, -1) for j in range(6)])


@pytest.mark.parametrize("n,budget", [(100000, 16384), (70001, 69999), (131072, 1)])
def test_long_requests(n, budget):
    check(n, [n, 10], [budget, 3], 4, 512, kv_heads=1, page=64)
    check(n, [n, 10], [budget, 3], 4, 0, kv_heads=1, page=64, accounts=lambda rng, s: rng.integers(0, 2, s))


def test_many_requests():
    rng = np.random.default_rng(9)
    check(9, rng.integers(0, 60, 400).tolist(), rng.integers(-1, 40, 400).tolist(), 1, 3, kv_heads=3)
