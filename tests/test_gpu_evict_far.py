"""Eviction and the choice of keys where they go ways of their own: more pages than fit beside the rows, tables with entries that are no page, more work than
a grid has workgroups, very long requests, and pools and accounts beyond 4 GiB."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import evict_reference as ev
from tests.test_gpu_page_evict import KINDS, Problem

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("stay", [65900, 65537, 30000])
def test_more_pages_than_are_kept_near(kind, stay):
    # 4096 pages of 16 keys and more, rows moving on both sides of the last one that fits; behind it a request whose pages do fit
    Problem(kind=kind, lengths=[66000, 700], stay=[stay, 333], page=16, kv_heads=1, seed=stay, spare=0).check()


def test_more_work_than_workgroups():
    rng = np.random.default_rng(2)
    lengths = rng.integers(0, 40, 11000)
    stay = (lengths * rng.random(11000)).astype(int)
    Problem(kind="fp8", lengths=lengths.tolist(), stay=stay.tolist(), kv_heads=2, seed=2).check()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("page,long", [(16, False), (64, False), (16, True)])
def test_entries_that_are_no_page(kind, page, long):
    """Keys on them move nowhere and nothing moves there; pages that go back are handed on as they are."""
    lengths, stay = ([66000], [65000]) if long else ([500, 300], [222, 299])
    p = Problem(kind=kind, lengths=lengths, stay=stay, page=page, kv_heads=2, seed=page, spare=9)
    bad = [(0, 1, -1), (0, 3, 1 << 30), (0, p.table.shape[1] - 3, -2 ** 31)] + ([(0, 4000, -1), (0, 4099, len(p.free))] if long else [(1, 0, 2 ** 31 - 1), (1, 4, -7)])
    for b, j, value in bad:
        p.table[b, j] = value
    none = lambda b, key: not 0 <= p.table[b, key // page] < len(p.free)
    k, v, w, kb, vb = p.device()
    want = [None if x is None else x.copy() for x in p.arrays]
    for b in range(len(lengths)):
        for g in range(2):
            for j, i in enumerate(p.kept[b, g, :stay[b]]):
                if j < i < lengths[b] and not none(b, i) and not none(b, j):
                    for x in want:
                        if x is not None:
                            x[p.table[b, j // page], j % page, g] = x[p.table[b, i // page], i % page, g]
    back = [p.table[b, j] for b in range(len(lengths)) for j in range(-(-stay[b] // page), -(-lengths[b] // page))]
    want_free = p.free.copy()
    want_free[p.n_free:p.n_free + len(back)] = back
    unit = 2 if kind == "mxfp4" else 1
    params = mp.make_paged_params(batch=len(lengths), n_q_heads=2, n_kv_heads=2, dtype="fp32" if kind == "fp32" else "bf16",
                                  kv_dtype=kind if kind in ("fp8", "mxfp4") else "", page_size=page, max_pages=p.table.shape[1], n_pages=len(p.free),
                                  k_strides=[unit * x for x in k.stride()[:3]], v_strides=[unit * x for x in v.stride()[:3]])
    free, n_free, status = i32(p.free), i32([p.n_free]), i32([9])
    mp.magicpig_page_evict(params, i32(p.kept), i32(lengths), i32(stay), i32(p.table), free, n_free, k, v, kb, vb, w, n_free, status)
    assert int(status) == 0 and int(n_free) == p.n_free + len(back)
    np.testing.assert_array_equal(free.cpu().numpy(), want_free)
    np.testing.assert_array_equal(w.view(torch.int32).cpu().numpy().transpose(0, 2, 1), want[2][..., 0])
    for got, x in zip((k, v, kb, vb), (want[0], want[1], want[3], want[4])):
        if x is not None:
            np.testing.assert_array_equal(got.contiguous().view(KINDS[kind][0] if x.shape[-1] > 4 else torch.uint8).cpu().numpy(), x)


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_pools_beyond_four_gigabytes(kind):
    page, n, stay = 16, 900, 500
    n_pages = (9 << 30) // (64 if kind == "mxfp4" else 256) // page
    held, rng = -(-n // page), np.random.default_rng(3)
    ids = np.array([n_pages - 1 - 11 * j if j % 2 else 5 * j for j in range(held)])
    at = torch.from_numpy(ids).cuda()
    width, dtype = (64, torch.uint8) if kind == "mxfp4" else (128, torch.bfloat16)
    make = lambda t, *shape: torch.empty(n_pages, *shape, dtype=t, device="cuda")
    arrays = [make(dtype, page, 1, width), make(dtype, page, 1, width), make(torch.float32, 1, page)]
    arrays += [make(torch.uint8, page, 1, 4), make(torch.uint8, page, 1, 4)] if kind == "mxfp4" else [None, None]
    kept = np.sort(rng.permutation(n)[:stay]).astype(np.int32)
    before = []
    for x in arrays:
        if x is not None:
            x[at] = torch.randint(0, 100, (held,) + x.shape[1:], device="cuda").to(x.dtype)
        before.append(None if x is None else x[at].reshape(held * page, -1).cpu())
    p = mp.make_paged_params(batch=1, n_q_heads=1, n_kv_heads=1, dtype="bf16", kv_dtype="mxfp4" if kind == "mxfp4" else "", page_size=page, max_pages=held,
                             n_pages=n_pages)
    free, n_free, status = torch.empty(n_pages, dtype=torch.int32, device="cuda"), i32([0]), i32([9])
    k, v, w, kb, vb = arrays
    mp.magicpig_page_evict(p, i32(kept[None, None]), i32([n]), i32([stay]), i32(ids[None]), free, n_free, k, v, kb, vb, w, n_free, status)
    assert int(status) == 0 and int(n_free) == held - -(-stay // page)
    np.testing.assert_array_equal(free[:int(n_free)].cpu().numpy(), ids[-(-stay // page):])
    for x, old in zip(arrays, before):
        if x is not None:
            want = old.clone()
            want[:stay] = old[torch.from_numpy(kept).long()]
            assert torch.equal(x[at].reshape(held * page, -1).cpu(), want)


def chosen(w, budget, first, last):
    """Keys of one head that stay, by a stable sort."""
    n = len(w)
    i = np.arange(n)
    sure = (i < first) | (i >= n - last)
    rank = np.where(sure, 0.0, np.where(np.isnan(w), 0.0, -w.astype(np.float64)))
    return np.sort(np.lexsort((i, rank, np.isnan(w), ~sure))[:budget])


def test_the_sort_chooses_as_the_plain_model_does():
    rng = np.random.default_rng(4)
    w = rng.integers(-2, 3, 300).astype(np.float32)
    w[rng.random(300) < 0.1] = np.nan
    kept, _ = ev.keep(w.reshape(1, 1, 300), np.zeros((1, 1), np.int32), [300], [77], 4, 9, 77)
    np.testing.assert_array_equal(kept[0, 0], chosen(w, 77, 4, 9))


@pytest.mark.parametrize("n,page", [(16 * 65280, 64), (16 * 65280 + 1, 64), (1200007, 1024)])
@pytest.mark.parametrize("few", [False, True])
def test_a_million_keys(n, page, few):
    # (several workgroups, and one where a part's counts would pass 16 bits; ranks of many kinds, and of three)
    rng = np.random.default_rng(n)
    pages = -(-n // page)
    w = rng.integers(0, 3, (pages, 1, page)).astype(np.float32) if few else rng.standard_normal((pages, 1, page)).astype(np.float32)
    table, budget = rng.permutation(pages), n // 3
    p = mp.make_paged_params(batch=1, n_q_heads=1, n_kv_heads=1, dtype="bf16", page_size=page, max_pages=pages, n_pages=pages)
    kept, out = torch.zeros(1, 1, budget, dtype=torch.int32, device="cuda"), i32([0])
    mp.magicpig_page_keep(p, torch.from_numpy(w).cuda(), i32(table[None]), i32([n]), i32([budget]), 5, 700, kept, out, mp.alloc_paged_workspace(p))
    assert int(out) == budget
    np.testing.assert_array_equal(kept[0, 0].cpu().numpy(), chosen(w[table].reshape(-1)[:n], budget, 5, 700))


@pytest.mark.parametrize("n", [3000, 50000])
def test_accounts_beyond_four_gigabytes(n):
    page, rng = 16, np.random.default_rng(n)
    n_pages, held = (5 << 30) // (2 * page * 4), -(-n // page)
    ids = np.array([n_pages - 1 - 11 * j if j % 2 else 5 * j for j in range(held)])
    w = rng.standard_normal((held, 2, page)).astype(np.float32)
    accounts = torch.empty(n_pages, 2, page, device="cuda")
    accounts[torch.from_numpy(ids).cuda()] = torch.from_numpy(w).cuda()
    p = mp.make_paged_params(batch=1, n_q_heads=2, n_kv_heads=2, dtype="bf16", page_size=page, max_pages=held, n_pages=n_pages)
    kept, out = torch.zeros(1, 2, 1000, dtype=torch.int32, device="cuda"), i32([0])
    mp.magicpig_page_keep(p, accounts, i32(ids[None]), i32([n]), i32([1000]), 4, 64, kept, out, mp.alloc_paged_workspace(p))
    for g in range(2):
        np.testing.assert_array_equal(kept[0, g].cpu().numpy(), chosen(w[:, g].reshape(-1)[:n], 1000, 4, 64))
