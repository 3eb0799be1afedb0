"""Accounts of attention weight against their definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import evict_reference as ev
from tests import mxfp_reference as mx
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
D = 128
KINDS = ["bf16", "fp32", "fp8", "mxfp4"]


class Problem:
    """A paged cache with random keys in the slots that requests hold and NaN in all others; accounts are random everywhere."""

    def __init__(self, *, kind, heads, kv_heads, page, lengths, new=None, layout="token", n_sink=0, n_local=0, scale=0.0, seed=0, spread=1.0,
                 spare_rows=0, bad=(), counted=None, table_width=0):
        rng = np.random.default_rng(seed)
        self.kind, self.page, self.lengths, self.n_sink, self.n_local, self.scale, self.layout = kind, page, lengths, n_sink, n_local, scale, layout
        batch = len(lengths)
        held = [-(-n // page) for n in lengths]
        max_pages, n_pages = max(max(max(held), 1) + 1, table_width), sum(held) + 3
        ids = rng.permutation(n_pages)[:sum(held)]
        self.table = np.full((batch, max_pages), -1, np.int32)
        used, at = np.zeros((n_pages, page), bool), 0
        for b, h in enumerate(held):
            self.table[b, :h] = ids[at:at + h]
            at += h
            i = np.arange(lengths[b])
            used[self.table[b, i // page], i % page] = True
        new = [1] * batch if new is None else new
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        tokens = int(self.start[-1]) + spare_rows
        k = np.where(used[:, :, None, None], rng.standard_normal((n_pages, page, kv_heads, D)) + rng.standard_normal((kv_heads, D)), np.nan)
        self.ks = self.kb = None
        if kind == "mxfp4":
            self.k, self.kb = (torch.from_numpy(x) for x in mx.quantise(k))
        elif kind == "fp8":
            self.k = torch.from_numpy(np.clip(40 * k, -448, 448)).float().to(torch.float8_e4m3fn)
            self.ks = torch.from_numpy(0.01 + 0.03 * rng.random(kv_heads)).float()
        else:
            self.k = torch.from_numpy(k).float().to(torch.bfloat16 if kind == "bf16" else torch.float32)
        self.q = torch.from_numpy(spread * rng.standard_normal((tokens, heads, D))).to(torch.float32 if kind == "fp32" else torch.bfloat16)
        for b, j, value in bad:
            self.table[b, j] = value
        self.heads, self.kv_heads, self.counted = heads, kv_heads, counted
        self.single = all(n == 1 for n in new) and spare_rows == 0
        self.max_new = max(max(new), 1)
        self.accounts = torch.from_numpy(rng.random((n_pages, kv_heads, page)).astype(np.float32))
        # the attention's own log-sum-exp, as it comes in float32
        self.lse = torch.from_numpy(np.nan_to_num(ref.attention(
            self.q.double().numpy(), self.keys(), np.zeros(self.keys().shape), self.table, lengths, None if self.single else self.start, n_sink, n_local,
            scale or None)[1], nan=7.0, neginf=-np.inf)).float()
        self.upload()

    def keys(self):
        if self.kind == "mxfp4":
            return mx.values(self.k.numpy(), self.kb.numpy())
        k = self.k.double().numpy()
        return k if self.ks is None else k * self.ks.double().numpy()[:, None]

    def upload(self):
        def pool(x):
            if x is None:
                return None
            if self.layout == "head":
                return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            if self.layout == "wide":                     # rows twice as long
                return torch.cat([x, x], -1).cuda()[..., :x.shape[-1]]
            return x.cuda()
        self.dk, self.dkb = pool(self.k), pool(self.kb)
        self.dq, self.dlse = self.q.cuda(), self.lse.cuda()
        i32 = lambda x: None if x is None else torch.from_numpy(np.asarray(x, np.int32)).cuda()
        self.dtable, self.dlen, self.dstart, self.dcounted = i32(self.table), i32(self.lengths), i32(self.start), i32(self.counted)
        self.dks = None if self.ks is None else self.ks.cuda()

    def params(self, **more):
        unit = 2 if self.kind == "mxfp4" else 1
        return mp.make_paged_params(**{**dict(
            batch=len(self.lengths), n_q_heads=self.heads, n_kv_heads=self.kv_heads, dtype="fp32" if self.kind == "fp32" else "bf16",
            kv_dtype=self.kind if self.kind in ("fp8", "mxfp4") else "", page_size=self.page, max_pages=self.table.shape[1], n_pages=self.k.shape[0],
            max_tokens=self.q.shape[0], max_new=self.max_new, n_sink=self.n_sink, n_local=self.n_local, scale=self.scale,
            k_strides=[unit * x for x in self.dk.stride()[:3]], q_strides=self.dq.stride()[:2]), **more})

    def call(self, p, accounts, ws, with_start=None):
        start = self.dstart if (not self.single if with_start is None else with_start) else None
        mp.magicpig_page_weights(p, self.dq, self.dk, self.dks, self.dkb, self.dtable, self.dlen, start, self.dlse, self.dcounted, accounts, ws)

    def run(self, with_start=None):
        p, accounts = self.params(), self.accounts.cuda()
        self.call(p, accounts, mp.alloc_paged_workspace(p), with_start)
        return accounts.cpu().double().numpy()

    def reference(self):
        return ev.weights(self.q.double().numpy(), self.keys(), self.table, self.lengths, None if self.single else self.start, self.lse.double().numpy(),
                          self.counted, self.accounts.double().numpy(), self.n_sink, self.n_local, self.scale or None)

    def check(self, with_start=None):
        self.compare(self.run(with_start))

    def compare(self, got):
        want, off = self.reference()
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        np.testing.assert_array_equal(got[np.isinf(want)], want[np.isinf(want)])
        fine = np.isfinite(want)
        d = np.abs(got - want)
        assert (d[fine] <= off[fine] + 1e-38).all(), (np.nanmax((d / (off + 1e-38))[fine]), np.argwhere(fine & (d > off + 1e-38))[:4])


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 300]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (3, 3), (16, 1), (64, 16)])
@pytest.mark.parametrize("page,layout", [(16, "token"), (64, "head"), (256, "wide")])
def test_one_token_per_request(kind, heads, kv_heads, page, layout):
    Problem(kind=kind, heads=heads, kv_heads=kv_heads, page=page, lengths=EDGES, layout=layout, seed=page + heads).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,kv_heads", [(20, 1), (64, 1), (128, 2), (21, 1)])
def test_many_heads_per_kv_head(kind, heads, kv_heads):
    Problem(kind=kind, heads=heads, kv_heads=kv_heads, page=32, lengths=[40, 0, 513], seed=heads).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", [[20011], [5000, 3, 9000, 0, 700]])
def test_long_caches(kind, lengths):
    Problem(kind=kind, heads=8, kv_heads=2, page=64, lengths=lengths, seed=3).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,kv_heads,new", [(8, 2, [4, 1, 3, 0, 2]), (10, 2, [6, 6, 2, 5, 1]), (4, 4, [1, 9, 16, 0, 33]),
                                                (8, 2, [70, 1, 33, 0, 8]), (16, 1, [40, 1, 1, 200, 5]), (7, 1, [5, 150, 3, 3, 333])])
def test_several_tokens(kind, heads, kv_heads, new):
    # (more new tokens than cached keys too: the first ones attend nothing)
    Problem(kind=kind, heads=heads, kv_heads=kv_heads, page=16, lengths=[70, 2, 33, 5, 530], new=new, spare_rows=2, seed=7).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("table_width", [60, 200, 700])
@pytest.mark.parametrize("heads,kv_heads,new,n_local", [(32, 8, [50, 33], 0), (24, 8, [44, 50], 100), (40, 8, [1, 40], 0)])
def test_many_rows_in_tables_of_many_widths(kind, table_width, heads, kv_heads, new, n_local):
    # (the more keys the tables have room for the fewer wavefronts split a tile's rows)
    Problem(kind=kind, heads=heads, kv_heads=kv_heads, page=32, lengths=[333, 700], new=new, n_local=n_local, n_sink=5 if n_local else 0,
            table_width=table_width, seed=table_width).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n_sink,n_local", [(0, 1), (4, 20), (0, 64), (40, 33), (100, 7), (70, 130), (5, 1 << 30), (1 << 30, 3)])
@pytest.mark.parametrize("new", [None, [1, 5, 0, 2, 8, 1], [1, 90, 0, 33, 64, 200]])
def test_sink_and_window(kind, n_sink, n_local, new):
    Problem(kind=kind, heads=6, kv_heads=2, page=32, lengths=[1, 95, 0, 34, 257, 700], new=new, n_sink=n_sink, n_local=n_local,
            spare_rows=1 if new else 0, seed=n_sink + n_local % 1000).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("counted", [[0, 0, 0, 0, 0, 0], [1, 70, 5, 30, 257, 100], [-5, 2 ** 31 - 1, -2 ** 31, 34, 200, 699]])
@pytest.mark.parametrize("new,n_local", [(None, 0), ([1, 0, 0, 2, 8, 1], 0), ([1, 0, 0, 2, 8, 1], 10), ([1, 90, 0, 0, 64, 200], 30)])
def test_accounts_that_begin_elsewhere(kind, counted, new, n_local):
    Problem(kind=kind, heads=4, kv_heads=2, page=16, lengths=[1, 95, 0, 34, 257, 700], new=new, n_local=n_local, n_sink=3 if n_local else 0, counted=counted,
            seed=8, spare_rows=1 if new else 0).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [None, [3, 2, 4], [50, 9, 64]])
def test_table_entries_that_are_no_page(kind, new):
    bad = [(0, 1, -1), (0, 2, 1 << 30), (1, 0, -2 ** 31), (2, 3, 2 ** 31 - 1), (2, 0, 10 ** 6)]
    Problem(kind=kind, heads=4, kv_heads=2, page=16, lengths=[90, 12, 64], new=new, bad=bad, seed=5, spare_rows=1 if new else 0).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,n_local", [([1, 1, 1], 0), ([4, 4, 4], 0), ([2, 2, 2], 6), ([40, 33, 40], 9)])
def test_nan_and_infinite_keys_stay_with_themselves(kind, new, n_local):
    p = Problem(kind=kind, heads=8, kv_heads=2, page=16, lengths=[80, 33, 40], new=new, n_local=n_local, n_sink=1 if n_local else 0, seed=9)
    def place(b, pos):
        return int(p.table[b, pos // 16]), pos % 16
    for b, pos, value in [(0, 5, float("nan")), (0, 79, float("nan")), (1, 30, float("-inf")), (2, 0, float("inf"))]:
        pg, at = place(b, pos)
        if kind == "mxfp4":
            p.kb[pg, at, 0, 1] = 255
        else:
            p.k[pg, at, 0, 40] = float("nan") if kind == "fp8" else value
    p.upload()
    p.check()


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_attend_nothing_and_lse_of_any_kind(kind):
    p = Problem(kind=kind, heads=4, kv_heads=1, page=16, lengths=[80, 300, 40], new=[4, 4, 4], seed=11)
    p.lse[0] = -float("inf")
    p.lse[5, 1] = float("inf")
    p.lse[6, 3] = -200.0                                   # (weights beyond float32: infinities)
    p.lse[11] = float("nan")
    p.upload()
    with np.errstate(over="ignore", invalid="ignore"):
        want, _ = p.reference()
        want = want.astype(np.float32)
    got = p.run()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    np.testing.assert_allclose(got[fine], want[fine], rtol=2e-5)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scale", [-0.5, 1e-30, 0.3])
def test_scales(kind, scale):
    for new in (None, [20, 33]):
        p = Problem(kind=kind, heads=4, kv_heads=2, page=16, lengths=[300, 40], new=new, scale=scale, seed=2)
        if kind == "fp8":
            p.ks = torch.tensor([-0.02, 0.0])
        p.upload()
        p.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,longest", [(333, 90), (1000, 3), (70, 2000)])
def test_many_requests(kind, batch, longest):
    rng = np.random.default_rng(batch)
    lengths = rng.integers(0, longest, batch).tolist()
    new = None if batch != 70 else rng.integers(0, 4, batch).tolist()
    Problem(kind=kind, heads=4, kv_heads=2, page=16, lengths=lengths, new=new, seed=1).check()


@pytest.mark.parametrize("kind", KINDS)
def test_strided_queries_either_form_and_the_same_bits(kind):
    p = Problem(kind=kind, heads=8, kv_heads=2, page=16, lengths=[3000, 40, 1], seed=4)
    wide = torch.full((3, 13, D), float("nan"), dtype=p.q.dtype, device="cuda")
    wide[:, 2:10] = p.dq
    a = p.run(False)
    p.dq = wide[:, 2:10]
    for with_start in (False, True):
        np.testing.assert_array_equal(p.run(with_start), a)
    many = Problem(kind=kind, heads=8, kv_heads=2, page=16, lengths=[3000, 400], new=[200, 333], seed=4)
    first = many.run()
    for _ in range(4):
        np.testing.assert_array_equal(many.run(), first)


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
@pytest.mark.parametrize("new", [1, 50])
def test_far_pools(kind, new):
    heads, page, n = 2, 16, 700
    small = Problem(kind=kind, heads=heads, kv_heads=1, page=page, lengths=[n], new=[new], seed=24)
    n_pages = (9 << 30) // (64 if kind == "mxfp4" else 256) // page
    held = -(-n // page)
    ids = torch.tensor([n_pages - 1 - 7 * j for j in range(held)], device="cuda")
    far = []
    for x in (small.k, small.kb):
        if x is not None:
            pool = torch.empty((n_pages, page, 1, x.shape[-1]), dtype=x.dtype, device="cuda")
            pool[ids] = x[torch.from_numpy(small.table[0, :held]).long()].cuda()
            far.append(pool)
    accounts = torch.empty(n_pages, 1, page, device="cuda")
    accounts[ids] = small.accounts[torch.from_numpy(small.table[0, :held]).long()].cuda()
    p = small.params(n_pages=n_pages, max_pages=held)
    start = None if new == 1 else small.dstart
    mp.magicpig_page_weights(p, small.dq, far[0], None, far[1] if kind == "mxfp4" else None, ids.to(torch.int32)[None].contiguous(), small.dlen, start,
                             small.dlse, None, accounts, mp.alloc_paged_workspace(p))
    got = small.accounts.double().numpy().copy()
    got[small.table[0, :held]] = accounts[ids].cpu().double().numpy()
    small.compare(got)
