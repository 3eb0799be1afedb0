"""Requests that share the pages of a prompt's beginning: accounts of all other pages, and eviction behind the shared keys."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import evict_reference as ev
from tests.test_gpu_page_weights import Problem

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.mark.parametrize("new", [None, [3, 1, 4, 2], [60, 1, 70, 33]])
@pytest.mark.parametrize("shared", [1, 5])
def test_what_is_shared_touches_nothing_else(shared, new):
    lengths = [300, 97, 230, 120]
    make = lambda bad: Problem(kind="bf16", heads=8, kv_heads=2, page=PAGE, lengths=lengths, new=new, seed=shared, bad=bad)
    common = make(()).table[0, :shared]
    p = make([(b, j, int(common[j])) for b in range(1, 4) for j in range(shared)])
    ours = np.ones(p.accounts.shape[0], bool)
    ours[common] = False
    accounts = p.accounts.cuda()
    params = p.params()
    ws = mp.alloc_paged_workspace(params)
    p.call(params, accounts, ws)
    got = accounts.cpu().double().numpy()
    want, _ = p.reference()
    p.compare(np.where(ours[:, None, None], got, want))
    # the first keys cover what is shared: their accounts play no part, and their rows stay
    budgets, first, last = [100, 90, 200, 81], shared * PAGE, 1
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    kept, stay = torch.zeros(4, 2, 200, dtype=torch.int32, device="cuda"), i32([0] * 4)
    mp.magicpig_page_keep(params, accounts, p.dtable, p.dlen, i32(budgets), first, last, kept, stay, ws)
    want_kept, want_stay = ev.keep(got.astype(np.float32), p.table, lengths, budgets, first, last, 200)
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    np.testing.assert_array_equal(stay.cpu().numpy(), want_stay)
    n_pages = ours.size
    k, v, free, n_free, status = p.dk, p.dk.flip(0).contiguous(), i32([0] * n_pages), i32([0]), i32([9])
    bits = lambda x: x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32).cpu().numpy().copy()
    arrays = [bits(k), bits(v), bits(accounts).transpose(0, 2, 1)]
    mp.magicpig_page_evict(params, kept, p.dlen, stay, p.dtable, free, n_free, k, v, None, None, accounts, n_free, status, ws)
    want_free, want_n, _ = ev.evict(want_kept, lengths, want_stay, p.table, np.zeros(n_pages, np.int32), 0, PAGE, arrays)
    assert int(status) == 0 and int(n_free) == want_n
    np.testing.assert_array_equal(free.cpu().numpy(), want_free)
    for a, b in zip((bits(k), bits(v), bits(accounts).transpose(0, 2, 1)), arrays):
        np.testing.assert_array_equal(a, b)
