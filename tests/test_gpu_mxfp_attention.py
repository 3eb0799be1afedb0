"""Exact attention over pools in four bits against its definition in 64 bits, for the values that the pools hold."""
import numpy as np
import pytest
import torch

from paper_2410_16179_amd import binding as mp
from tests import mxfp_reference as mx
from tests import paged_reference as ref

pytestmark = pytest.mark.gpu
D = 128


class Problem:
    """A paged cache in four bits with random keys in the slots that requests hold and NaN in all others."""

    def __init__(self, *, heads, kv_heads, page, lengths, new=None, layout="token", n_sink=0, n_local=0, scale=0.0, seed=0, spread=1.0,
                 spare_rows=0, bad=(), size=1.0):
        rng = np.random.default_rng(seed)
        self.page, self.lengths, self.n_sink, self.n_local, self.scale = page, lengths, n_sink, n_local, scale
        batch = len(lengths)
        held = [-(-n // page) for n in lengths]
        max_pages, n_pages = max(max(held), 1) + 1, sum(held) + 3
        ids = rng.permutation(n_pages)[:sum(held)]
        self.table = np.full((batch, max_pages), -1, np.int32)
        at = 0
        used = np.zeros((n_pages, page), bool)
        for b, h in enumerate(held):
            self.table[b, :h] = ids[at:at + h]
            at += h
            i = np.arange(lengths[b])
            used[self.table[b, i // page], i % page] = True
        new = [1] * batch if new is None else new
        self.start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        tokens = int(self.start[-1]) + spare_rows
        shift = rng.standard_normal((kv_heads, D))
        channel = np.exp(0.7 * rng.standard_normal((kv_heads, D)))
        pool = lambda more: mx.quantise(np.where(used[:, :, None, None], size * channel * (rng.standard_normal((n_pages, page, kv_heads, D)) + more), np.nan))
        self.k, self.kb = pool(shift)
        self.v, self.vb = pool(0.2)
        self.q = torch.from_numpy(spread / size * rng.standard_normal((tokens, heads, D))).to(torch.bfloat16)
        for b, j, value in bad:
            self.table[b, j] = value
        self.heads, self.kv_heads, self.layout = heads, kv_heads, layout
        self.single = all(n == 1 for n in new) and spare_rows == 0
        self.max_new = max(max(new), 1)
        self.upload()

    def upload(self):
        def pool(x):
            x = torch.from_numpy(x)
            if self.layout == "head":
                return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            if self.layout == "wide":                     # rows of 256 elements, the others NaN
                return torch.cat([x, torch.full_like(x, 255)], -1).cuda()[..., :x.shape[-1]]
            return x.cuda()
        self.dk, self.dv, self.dkb, self.dvb = (pool(x) for x in (self.k, self.v, self.kb, self.vb))
        self.dq = self.q.cuda()
        self.dtable, self.dlen, self.dstart = (torch.from_numpy(np.asarray(x, np.int32)).cuda() for x in (self.table, self.lengths, self.start))

    def params(self, **more):
        return mp.make_paged_params(**{**dict(
            batch=len(self.lengths), n_q_heads=self.heads, n_kv_heads=self.kv_heads, dtype="bf16", kv_dtype="mxfp4", page_size=self.page,
            max_pages=self.table.shape[1], n_pages=self.k.shape[0], max_tokens=self.q.shape[0], max_new=self.max_new, n_sink=self.n_sink,
            n_local=self.n_local, scale=self.scale, k_strides=[2 * x for x in self.dk.stride()[:3]], v_strides=[2 * x for x in self.dv.stride()[:3]],
            q_strides=self.dq.stride()[:2]), **more})

    def call(self, p, out, lse, ws, with_start=None):
        start = self.dstart if (not self.single if with_start is None else with_start) else None
        mp.magicpig_paged_attention_mxfp(p, self.dq, self.dk, self.dv, self.dkb, self.dvb, self.dtable, self.dlen, start, out, lse, ws)

    def outputs(self):
        out = torch.full((self.q.shape[0], self.heads, D), 7.0, dtype=torch.bfloat16, device="cuda")
        return out, torch.full(out.shape[:2], 7.0, device="cuda")

    def run(self, with_start=None):
        p = self.params()
        out, lse = self.outputs()
        self.call(p, out, lse, mp.alloc_paged_workspace(p), with_start)
        torch.cuda.synchronize()
        return out.cpu().double().numpy(), lse.cpu().double().numpy()

    def reference(self):
        return ref.attention(self.q.double().numpy(), mx.values(self.k, self.kb), mx.values(self.v, self.vb), self.table, self.lengths,
                             None if self.single else self.start, self.n_sink, self.n_local, self.scale or None, self.max_new)

    def check(self, with_start=None):
        self.compare(*self.run(with_start))

    def compare(self, out, lse):
        want, want_lse, size, reach, count = self.reference()
        real = np.zeros(want_lse.shape, bool)
        for b in range(len(self.lengths)):
            real[self.start[b]:self.start[b + 1]] = True
        np.testing.assert_array_equal(out[~real], 7.0)    # rows of no request
        np.testing.assert_array_equal(lse[~real], 7.0)
        np.testing.assert_array_equal(np.isnan(out[real]), np.isnan(want[real]))
        # (the pools' values are bf16 exactly, and the weights the sum of two bf16)
        tol = ref.tolerance(want, size, reach, count, "bf16", False)
        fine = real[..., None] & np.isfinite(want)
        off = np.abs(out - want)
        assert (off[fine] <= tol[fine]).all(), (np.nanmax((off / tol)[fine]), np.argwhere(fine & (off > tol))[:4])
        fine = real & np.isfinite(want_lse)
        np.testing.assert_array_equal(lse[real & (want_lse == -np.inf)], -np.inf)
        off = np.abs(lse - want_lse)
        assert (off[fine] <= ref.lse_tolerance(want_lse, reach, count)[fine]).all(), np.nanmax(off[fine])


EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 300]


@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (3, 3), (10, 2), (16, 1)])
@pytest.mark.parametrize("page,layout", [(16, "token"), (64, "head"), (32, "wide"), (256, "token")])
def test_one_token_per_request(heads, kv_heads, page, layout):
    Problem(heads=heads, kv_heads=kv_heads, page=page, lengths=EDGES, layout=layout, seed=page + heads).check()


@pytest.mark.parametrize("page", [128, 1024])
@pytest.mark.parametrize("new", [None, [5, 1, 3], [60, 1, 64]])
def test_large_pages(page, new):
    Problem(heads=8, kv_heads=2, page=page, lengths=[2100, 1, 1024], new=new, n_local=0, seed=page).check()
    Problem(heads=8, kv_heads=2, page=page, lengths=[2100, 1, 1024], new=new, n_sink=70, n_local=300, seed=page).check()


@pytest.mark.parametrize("heads,kv_heads", [(20, 1), (64, 1), (128, 2)])
def test_more_heads_per_kv_head_than_a_tile_has_rows(heads, kv_heads):
    Problem(heads=heads, kv_heads=kv_heads, page=32, lengths=[40, 0, 513], seed=heads).check()


@pytest.mark.parametrize("lengths", [[20011], [5000, 3, 9000, 0, 700]])
def test_long_caches_cut_into_pieces(lengths):
    Problem(heads=8, kv_heads=2, page=64, lengths=lengths, seed=3).check()


@pytest.mark.parametrize("heads,kv_heads,new", [(8, 2, [4, 1, 3, 0, 2]), (10, 2, [6, 6, 2, 5, 1]), (4, 4, [1, 9, 16, 0, 33]),
                                                (8, 2, [70, 1, 33, 0, 8]), (16, 1, [40, 1, 1, 200, 5])])
def test_new_tokens_attend_causally(heads, kv_heads, new):
    # (more new tokens than cached keys too: the first ones attend nothing)
    Problem(heads=heads, kv_heads=kv_heads, page=16, lengths=[70, 2, 33, 5, 530], new=new, spare_rows=2, seed=7).check()


@pytest.mark.parametrize("layout,page", [("token", 16), ("wide", 128), ("head", 32)])
@pytest.mark.parametrize("lengths,new,n_local", [([6000, 300, 1030], [150, 40, 129], 0), ([6000, 300, 1030], [150, 40, 129], 700), ([515], [515], 0)])
def test_chunks_of_prompts(layout, page, lengths, new, n_local):
    Problem(heads=4, kv_heads=1, page=page, layout=layout, lengths=lengths, new=new, n_local=n_local, n_sink=3 if n_local else 0,
            spare_rows=1, seed=12).check()


@pytest.mark.parametrize("n_sink,n_local", [(0, 1), (4, 20), (0, 64), (40, 33), (100, 7), (70, 130), (5, 1 << 30), (1 << 30, 3)])
@pytest.mark.parametrize("new", [None, [1, 5, 0, 2, 8, 1], [1, 90, 0, 33, 64, 200]])
def test_sink_and_window(n_sink, n_local, new):
    Problem(heads=6, kv_heads=2, page=32, lengths=[1, 95, 0, 34, 257, 700], new=new, n_sink=n_sink, n_local=n_local,
            spare_rows=1 if new else 0, seed=n_sink + n_local % 1000).check()


@pytest.mark.parametrize("new", [None, [3, 2, 4], [50, 9, 64]])
def test_table_entries_that_are_no_page(new):
    bad = [(0, 1, -1), (0, 2, 1 << 30), (1, 0, -2 ** 31), (2, 3, 2 ** 31 - 1), (2, 0, 10 ** 6)]
    Problem(heads=4, kv_heads=2, page=16, lengths=[90, 12, 64], new=new, bad=bad, seed=5, spare_rows=1 if new else 0).check()


@pytest.mark.parametrize("new,n_local", [([5, 4, 3], 0), ([5, 4, 3], 6), ([60, 33, 40], 0), ([60, 33, 40], 9), ([1, 1, 1], 0)])
def test_nan_blocks_reach_the_rows_that_attend_them_alone(new, n_local):
    p = Problem(heads=4, kv_heads=2, page=16, lengths=[80, 33, 40], new=new, n_local=n_local, n_sink=1 if n_local else 0, seed=9)

    def place(b, pos):
        return int(p.table[b, pos // 16]), pos % 16
    for b, pos, block in [(0, 78, 0), (0, 75, 3), (1, 30, 2), (2, 39, 0), (2, 36, 1)]:
        pg, at = place(b, pos)
        p.vb[pg, at, b % 2, block] = 255
    pg, at = place(1, 32)
    p.kb[pg, at, 0, 1] = 255                              # the last key of request 1: its row alone
    p.upload()
    p.check()


def test_logits_beyond_the_exponential_s_range():
    for new in (None, [40, 40]):
        Problem(heads=4, kv_heads=2, page=16, lengths=[300, 40], new=new, spread=100.0, seed=2).check()
        Problem(heads=4, kv_heads=2, page=16, lengths=[300, 40], new=new, scale=-0.7, spread=2.0, seed=2).check()


@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 60])
@pytest.mark.parametrize("new", [None, [40, 33]])
def test_keys_and_values_of_any_size(size, new):
    Problem(heads=4, kv_heads=2, page=16, lengths=[300, 40], new=new, size=size, seed=4).check()


@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("heads,kv_heads,batch,longest", [(32, 32, 70, 60), (16, 8, 300, 40), (24, 12, 200, 90), (64, 32, 140, 150)])
def test_many_short_requests(layout, heads, kv_heads, batch, longest):
    # workgroups take two, four or eight KV heads at once
    lengths = np.random.default_rng(batch).integers(0, longest, batch).tolist()
    new = None if heads > 24 else [1 + i % 4 for i in range(batch)]
    Problem(heads=heads, kv_heads=kv_heads, page=16, lengths=lengths, new=new, layout=layout, seed=batch).check()


@pytest.mark.parametrize("heads,kv_heads,new,shortest", [(32, 8, 1, 7000), (16, 8, 1, 7000), (32, 8, 4, 6000), (48, 12, 1, 1)])
def test_long_requests_over_neighbouring_heads(heads, kv_heads, new, shortest):
    # items that are cut, in sets of KV heads whose rows are neighbours; all requests share the longest one's pages
    batch, longest = (20, 8000) if shortest > 1 else (90, 9000)
    lengths = [longest] + np.random.default_rng(26).integers(shortest, longest, batch - 1).tolist()
    p = Problem(heads=heads, kv_heads=kv_heads, page=64, lengths=[longest] + [0] * (batch - 1), new=[new] * batch, seed=26)
    p.lengths = lengths
    p.table[1:] = p.table[0]
    p.upload()
    p.check()


@pytest.mark.parametrize("how", [dict(lengths=[30000, 700]), dict(lengths=[9000, 9001, 40]), dict(lengths=[6000, 900], new=[120, 64])])
def test_the_same_bits_every_time(how):
    p = Problem(heads=8, kv_heads=2, page=32, seed=23, **how)
    first = p.run()
    for _ in range(5):
        again = p.run()
        np.testing.assert_array_equal(first[0], again[0])
        np.testing.assert_array_equal(first[1], again[1])


def test_either_form_of_single_tokens():
    p = Problem(heads=8, kv_heads=2, page=16, lengths=[300, 40, 1], seed=4)
    a, b = p.run(False), p.run(True)
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(a[1], b[1])


@pytest.mark.parametrize("new", [None, [3, 40]])
def test_the_same_as_the_rows_read_back_in_bf16(new):
    # the definition's other half: attention over what the read gives
    p = Problem(heads=8, kv_heads=2, page=16, lengths=[2000, 77], new=new, seed=31)
    n_pages, page = p.k.shape[:2]
    k, v = (torch.zeros(n_pages, page, 2, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = torch.arange(n_pages * page, device="cuda")
    every = p.params(max_tokens=n_pages * page, k_new_strides=(2 * D, D), v_new_strides=(2 * D, D))
    mp.magicpig_page_read_mxfp(every, p.dk, p.dv, p.dkb, p.dvb, slots, k, v)
    plain = p.params(kv_dtype="", k_strides=k.stride()[:3], v_strides=v.stride()[:3])
    out, lse = p.outputs()
    start = None if p.single else p.dstart
    mp.magicpig_paged_attention(plain, p.dq, k, v, None, None, p.dtable, p.dlen, start, out, lse, mp.alloc_paged_workspace(plain))
    p.compare(out.cpu().double().numpy(), lse.cpu().double().numpy())


@pytest.mark.parametrize("new", [1, 3, 40])
def test_far_pools(new):
    heads, page, n = 2, 16, 700
    n_pages = (9 << 30) // 64 // page
    small = Problem(heads=heads, kv_heads=1, page=page, lengths=[n], new=[new], seed=24)
    small.single = False
    held = -(-n // page)
    ids = torch.tensor([n_pages - 1 - 7 * j for j in range(held)], device="cuda")
    far = []
    for x in (small.k, small.v, small.kb, small.vb):
        pool = torch.empty(n_pages, page, 1, x.shape[-1], dtype=torch.uint8, device="cuda")
        pool[ids] = torch.from_numpy(x[small.table[0, :held]]).cuda()
        far.append(pool)
    p = small.params(n_pages=n_pages, max_pages=held)
    out, lse = small.outputs()
    mp.magicpig_paged_attention_mxfp(p, small.dq, *far, ids.to(torch.int32)[None].contiguous(), small.dlen, small.dstart, out, lse,
                                     mp.alloc_paged_workspace(p))
    small.compare(out.cpu().double().numpy(), lse.cpu().double().numpy())


@pytest.mark.parametrize("new", [None, [2, 1, 3], [40, 9, 64]])
def test_captured_and_replayed_with_other_lengths(new):
    p = Problem(heads=8, kv_heads=2, page=16, lengths=[900, 130, 64], new=new, seed=41, spare_rows=1 if new else 0)
    params = p.params()
    ws = mp.alloc_paged_workspace(params)
    out, lse = p.outputs()
    p.call(params, out, lse, ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        p.call(params, out, lse, ws)
    for lengths in ([900, 130, 64], [3, 0, 64], [333, 129, 1], [900, 130, 64]):
        p.lengths = lengths
        p.dlen.copy_(torch.tensor(lengths, dtype=torch.int32))
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        p.compare(out.cpu().double().numpy(), lse.cpu().double().numpy())


def test_on_another_stream_and_two_at_once():
    a, b = (Problem(heads=8, kv_heads=2, page=16, lengths=[5000 + i, 70], seed=50 + i) for i in range(2))
    made = [(p, p.params(), *p.outputs()) for p in (a, b)]
    spaces = [mp.alloc_paged_workspace(m[1]) for m in made]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(3):
        for (p, params, out, lse), ws, s in zip(made, spaces, streams):
            with torch.cuda.stream(s):
                p.call(params, out, lse, ws)
    torch.cuda.synchronize()
    for p, _, out, lse in made:
        p.compare(out.cpu().double().numpy(), lse.cpu().double().numpy())
