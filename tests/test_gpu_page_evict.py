"""Keys that stay move to the front and pages go back, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import evict_reference as ev

pytestmark = pytest.mark.gpu
KINDS = {"bf16": (torch.int16, 128), "fp32": (torch.int32, 128), "fp8": (torch.uint8, 128), "mxfp4": (torch.uint8, 64)}


class Problem:
    def __init__(self, *, kind, lengths, stay, kv_heads=2, page=16, layout="token", seed=0, max_keep=None, accounts=True, choose=None, spare=7):
        rng = np.random.default_rng(seed)
        self.kind, self.page, self.kv_heads, self.lengths, self.stay, self.layout = kind, page, kv_heads, lengths, stay, layout
        held = [-(-n // page) for n in lengths]
        max_pages, n_pages = max(max(held), 1) + 1, sum(held) + spare
        ids = rng.permutation(n_pages).astype(np.int32)
        self.table, at = np.full((len(lengths), max_pages), -1, np.int32), 0
        for b, h in enumerate(held):
            self.table[b, :h] = ids[at:at + h]
            at += h
        self.n_free = min(spare, 3)
        self.free = np.zeros(n_pages, np.int32)
        self.free[:self.n_free] = ids[at:at + self.n_free]
        max_keep = max(max(stay), 1) if max_keep is None else max_keep
        self.kept = np.full((len(lengths), kv_heads, max_keep), -1, np.int32)
        choose = choose or (lambda rng, n, m: np.sort(rng.permutation(n)[:m]))
        for b, (n, m) in enumerate(zip(lengths, stay)):
            if 0 <= m < n and m <= max_keep:
                for g in range(kv_heads):
                    self.kept[b, g, :m] = choose(rng, n, m)
        dtype, width = KINDS[kind]
        bits = lambda w, t: rng.integers(np.iinfo(t).min, np.iinfo(t).max, (n_pages, page, kv_heads, w), dtype=t, endpoint=True)
        np_type = {torch.int16: np.int16, torch.int32: np.int32, torch.uint8: np.uint8}[dtype]
        self.arrays = [bits(width, np_type), bits(width, np_type), bits(1, np.int32) if accounts else None]
        self.arrays += [bits(4, np.uint8), bits(4, np.uint8)] if kind == "mxfp4" else [None, None]
        self.accounts = accounts

    def device(self):
        def pool(x, view):
            if x is None:
                return None
            x = torch.from_numpy(x).view(view)
            if self.layout == "head":
                return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            if self.layout == "wide":
                return torch.cat([x, x], -1).cuda()[..., :x.shape[-1]]
            return x.cuda()
        real = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.uint8, "mxfp4": torch.uint8}[self.kind]
        k, v, w, kb, vb = self.arrays
        w = None if w is None else torch.from_numpy(w[..., 0]).view(torch.float32).permute(0, 2, 1).contiguous().cuda()
        return pool(k, real), pool(v, real), w, pool(kb, torch.uint8), pool(vb, torch.uint8)

    def check(self, with_kept=True, in_place=False, times=1):
        k, v, w, kb, vb = self.device()
        unit = 2 if self.kind == "mxfp4" else 1
        p = mp.make_paged_params(batch=len(self.lengths), n_q_heads=self.kv_heads, n_kv_heads=self.kv_heads, dtype="fp32" if self.kind == "fp32" else "bf16",
                                 kv_dtype=self.kind if self.kind in ("fp8", "mxfp4") else "", page_size=self.page, max_pages=self.table.shape[1],
                                 n_pages=len(self.free), k_strides=[unit * x for x in k.stride()[:3]], v_strides=[unit * x for x in v.stride()[:3]])
        i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
        free, n_free, status = i32(self.free), i32([self.n_free]), i32([77])
        n_out = n_free if in_place else i32([-1])
        kept, table = i32(self.kept) if with_kept else None, i32(self.table)
        for _ in range(times):
            mp.magicpig_page_evict(p, kept, i32(self.lengths), i32(self.stay), table, free, n_free, k, v, kb, vb, w, n_out, status,
                                   mp.alloc_paged_workspace(p))
        want = [None if x is None else x.copy() for x in self.arrays]
        for _ in range(times):
            want_free, want_n, want_status = ev.evict(self.kept if with_kept else None, self.lengths, self.stay, self.table, self.free, self.n_free, self.page,
                                                      [x for x in want if x is not None])
        assert int(status) == want_status and int(n_out) == want_n
        np.testing.assert_array_equal(free.cpu().numpy(), want_free)
        np.testing.assert_array_equal(table.cpu().numpy(), self.table)
        if w is not None:
            np.testing.assert_array_equal(w.view(torch.int32).cpu().numpy().transpose(0, 2, 1), want[2][..., 0])
        for got, x in zip((k, v, kb, vb), (want[0], want[1], want[3], want[4])):
            if x is not None:
                np.testing.assert_array_equal(got.contiguous().view(KINDS[self.kind][0] if x.shape[-1] > 4 else torch.uint8).cpu().numpy(), x)


LENGTHS = [0, 1, 16, 17, 100, 300, 300, 64, 900]
STAY = [0, 0, 15, 16, 100, 1, 299, 33, 450]


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("page,layout,kv_heads", [(16, "token", 2), (64, "head", 3), (32, "wide", 8), (1024, "token", 1)])
def test_rows_move_and_pages_go_back(kind, page, layout, kv_heads):
    Problem(kind=kind, lengths=LENGTHS, stay=STAY, page=page, layout=layout, kv_heads=kv_heads, seed=page).check()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("choose", [
    lambda rng, n, m: np.arange(n - m, n), lambda rng, n, m: np.arange(m), lambda rng, n, m: np.concatenate([np.arange(m - 1), [n - 1]]),
    lambda rng, n, m: np.concatenate([[0], np.arange(n - m + 1, n)]), lambda rng, n, m: np.linspace(0, n - 1, m).astype(int)])
def test_long_requests(kind, choose):
    # by one, by few, by half, and by nearly all
    for lengths, stay in (([5000, 3001], [4999, 1500]), ([9000], [8936]), ([20000], [700])):
        Problem(kind=kind, lengths=lengths, stay=stay, choose=choose, page=64, kv_heads=1, seed=5).check()


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_without_accounts_in_place_and_again(kind):
    Problem(kind=kind, lengths=LENGTHS, stay=STAY, accounts=False, seed=3).check(in_place=True)
    # (the same list again moves the rows again: nothing of the first call is kept)
    Problem(kind=kind, lengths=LENGTHS, stay=STAY, seed=4).check(times=2)


def test_only_lengths_shrink():
    Problem(kind="bf16", lengths=LENGTHS, stay=STAY, seed=6).check(with_kept=False)
    Problem(kind="bf16", lengths=[100, 90], stay=[99, 10], seed=6, max_keep=1).check(with_kept=False)


@pytest.mark.parametrize("how", [dict(stay=[10, 91]), dict(stay=[-1, 5]), dict(lengths=[-3, 90]), dict(stay=[50, 5], max_keep=49)])
def test_arguments_that_do_not_fit(how):
    p = Problem(kind="bf16", lengths=[100, 90], stay=[40, 5], seed=7)
    for name, value in how.items():
        if name == "max_keep":
            p.kept = np.ascontiguousarray(p.kept[..., :value])
        else:
            setattr(p, name, value)
    p.check()


def test_a_stack_beyond_its_end():
    p = Problem(kind="bf16", lengths=[100, 90], stay=[40, 5], seed=8, spare=2)
    p.n_free = len(p.free) - 3
    p.check()
    p.n_free = -1
    p.check()
    p.n_free = len(p.free) - (7 - 3) - (6 - 1)
    p.check()


def test_entries_that_do_not_ascend_move_nothing_out_of_place():
    p = Problem(kind="bf16", lengths=[300], stay=[40], kv_heads=1, seed=9)
    before = [x.copy() for x in p.arrays if x is not None]
    p.kept[0, 0, :40] = [0, 300, -1, 2, 2 ** 31 - 1, -2 ** 31] + [7] * 34
    k, v, w, _, _ = p.device()
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    params = mp.make_paged_params(batch=1, n_q_heads=1, n_kv_heads=1, dtype="bf16", page_size=16, max_pages=p.table.shape[1], n_pages=len(p.free))
    status = i32([5])
    mp.magicpig_page_evict(params, i32(p.kept), i32(p.lengths), i32(p.stay), i32(p.table), i32(p.free), i32([p.n_free]), k, v, None, None, w, i32([0]),
                           status)
    assert int(status) == 0
    got = k.view(torch.int16).cpu().numpy()
    # rows outside the first forty keys are as they were
    mine = np.zeros(got.shape[:2], bool)
    i = np.arange(40)
    mine[p.table[0, i // 16], i % 16] = True
    np.testing.assert_array_equal(got[~mine], before[0][~mine])


def test_many_requests():
    rng = np.random.default_rng(10)
    lengths = rng.integers(0, 70, 1500)
    stay = (lengths * rng.random(1500)).astype(int)
    Problem(kind="fp8", lengths=lengths.tolist(), stay=stay.tolist(), kv_heads=2, seed=10).check()
