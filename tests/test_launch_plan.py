"""The rules of csrc/launch_plan.h, compiled on their own."""
import ctypes
import math
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "launch_plan.h"
extern "C" {
void gather(int units, int G, long nblk, long n_static, int tau, int* got) {
  const mp::GatherPlan p = mp::plan_gather(units, G, nblk, n_static, tau);
  got[0] = p.run_blocks; got[1] = p.runs; got[2] = p.static_runs; got[3] = p.static_keys; got[4] = p.full;
}
long head_limit(int tuned, int G) { return mp::head_per_workgroup_limit(tuned, G); }
void paged(int batch, int kv, int group, int fp32, long max_tokens, int max_new, int starts, long max_len, int n_sink, int n_local, int row_bytes, long* got) {
  const mp::PagedForm f = mp::paged_form(batch, kv, group, fp32, max_tokens, max_new, starts, max_len, n_sink, n_local, row_bytes);
  const long all[] = {f.rows, f.key_tile, f.tile_tokens, f.head_blocks, f.target, f.min_tiles, f.near_shift, f.set_shift, f.group_shift, f.shares[0], f.shares[1], f.shares[2], f.shares[3], f.items, f.pieces,
                      f.units, f.slots};
  for (int i = 0; i < 17; ++i) got[i] = all[i];
}
int plan_workgroups(int batch, long max_tokens, int in_place) { return mp::page_plan_workgroups(batch, max_tokens, in_place); }
int hash_f32(int K, long groups32, long groups64) { return mp::hash_f32_keys(K, groups32, groups64); }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("plan")
    (tmp / "shim.cpp").write_text(SHIM)
    so = str(tmp / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2410_16179_amd", "csrc"), str(tmp / "shim.cpp"),
                    "-o", so], check=True)
    return ctypes.CDLL(so)


def gather(plan, units, G, n, n_static=68, tau=2):
    got = (ctypes.c_int * 5)()
    plan.gather(units, G, ctypes.c_long((n + 63) // 64), ctypes.c_long(n_static), tau, got)
    return tuple(got)


@pytest.mark.parametrize("units,G,n,n_static", [
    (64, 8, 1024, 1004), (64, 8, 2048, 68), (64, 8, 131072, 68), (8, 4, 16384, 4100), (8, 4, 16384, 16384), (1, 1, 64, 64), (64, 8, 65536, 6004),
    (80, 8, 10300, 700), (1, 4, 100000, 0), (512, 1, 4096, 516), (64, 8, 8192, 516), (260, 1, 200, 65)])
def test_gather_wavefronts_cover_the_blocks_and_share_the_static_set(plan, units, G, n, n_static):
    run_blocks, runs, own, keys, full = gather(plan, units, G, n, n_static)
    nblk = (n + 63) // 64
    assert run_blocks % 16 == 0 and run_blocks <= 128 and (runs - 1) * run_blocks < nblk <= runs * run_blocks
    assert full or run_blocks == 16                          # the form without full batches has a list for one piece
    # own wavefronts take the whole set; of keys dealt over the runs none gets more than two batches per piece, and no
    # more than half a batch where the runs leave the chip room
    if own:
        assert (own - 1) * keys < n_static <= own * keys and (full or keys == 32)
    else:
        share = -(-n_static // runs)
        assert share <= (64 * (run_blocks // 16) if units * runs * G >= 1024 else 16)
    # the partials fit the room that the workspace has for them
    assert runs + own <= -(-nblk // 16) + -(-n_static // 32)


def test_gather_forms_at_the_sizes_of_its_gpu_test(plan):
    # pieces of sixteen blocks per run, own static wavefronts and whether full batches have code of their own
    # (tests/test_gpu_gather_runs.py)
    def form(*a, **kw):
        run_blocks, _, own, keys, full = gather(plan, *a, **kw)
        return run_blocks // 16, (own, keys) if own else 0, bool(full)
    assert [form(64, 8, 10300), form(80, 5, 17000), form(128, 8, 35000)] == [(2, 0, True), (2, 0, True), (8, 0, True)]
    assert form(64, 8, 1000, 904) == (1, (15, 64), True)
    assert form(8, 4, 9000, 4131, tau=3) == (1, (65, 64), True)
    assert form(8, 4, 2500, 230, tau=3) == (1, (8, 32), False)
    assert form(8, 2, 3333, 3333, tau=3) == (1, (105, 32), False)
    assert form(260, 1, 200, 65) == (1, (3, 32), False)
    assert form(128, 8, 9000, 3000) == (3, (24, 128), True)
    assert form(8, 4, 16384, 68, tau=3) == (1, 0, False)


@pytest.mark.parametrize("K,groups32,keys", [
    (1, 256, 32), (2, 512, 32), (2, 1000, 32), (3, 2550, 32), (4, 257, 32), (4, 8192, 32),   # narrow tables: 32 throughout
    (5, 1002, 64), (8, 256, 32), (8, 384, 64), (8, 642, 32), (8, 1536, 64), (9, 760, 32), (10, 320, 64), (10, 515, 32), (10, 770, 64),
    (10, 2560, 64), (16, 258, 64), (16, 750, 32)])
def test_keys_of_a_float32_hashing_workgroup(plan, K, groups32, keys):
    # the faster of the two forms where they differ by more than a tenth; either where they do not
    assert plan.hash_f32(K, ctypes.c_long(groups32), ctypes.c_long((groups32 + 1) // 2)) == keys


@pytest.mark.parametrize("units,G,n,tuned,one", [
    # the sizes of tests/test_gpu_head_per_workgroup.py (up to 780 workgroups a run is four key blocks)
    (1, 4, 70, True, True), (8, 2, 1001, True, True), (8, 4, 2048, True, True), (8, 3, 1300, True, True), (2, 8, 4096, True, True), (4, 5, 777, True, True),
    (1, 7, 1500, False, True), (4, 3, 515, False, True), (8, 5, 1600, False, True), (8, 4, 6144, True, True), (8, 4, 6209, True, False), (1, 2, 3, True, True),
    # and those on which the limits rest
    (8, 2, 4096, True, True), (8, 2, 8192, True, False), (8, 2, 8192, False, False), (8, 3, 10000, True, False), (8, 4, 10000, True, False),
    (8, 4, 4096, False, True), (8, 4, 6144, False, False), (8, 5, 6400, True, True), (4, 7, 9000, True, True), (8, 8, 4000, False, True), (8, 8, 8000, True, False)])
def test_head_per_workgroup(plan, units, G, n, tuned, one):
    plan.head_limit.restype = ctypes.c_long
    assert (units * (-(-n // 256)) * G <= plan.head_limit(int(tuned), G)) == one


_PAGED = ("rows", "key_tile", "tile_tokens", "head_blocks", "target", "min_tiles", "near_shift", "set_shift", "group_shift", "shares0", "shares1", "shares2", "shares3", "items", "pieces", "units", "slots")


def paged(plan, batch, kv, group, fp32=False, max_tokens=None, max_new=1, starts=False, max_len=4096, n_sink=0, n_local=0, row_bytes=0):
    got = (ctypes.c_long * len(_PAGED))()
    plan.paged(batch, kv, group, int(fp32), ctypes.c_long(batch if max_tokens is None else max_tokens), max_new, int(starts), ctypes.c_long(max_len),
               n_sink, n_local, row_bytes, got)
    return dict(zip(_PAGED, got))


def test_rows_of_paged_attention_s_forms(plan):
    assert [paged(plan, 1, 8, g, max_new=t)["rows"] for g, t in [(1, 1), (4, 4), (16, 1), (4, 5), (32, 1), (5, 6), (4, 9), (64, 1)]] == \
        [16, 16, 16, 32, 32, 32, 128, 128]
    assert all(paged(plan, 1, 8, g, fp32=True, max_new=t)["rows"] == 16 for g, t in [(1, 1), (4, 100), (64, 1)])
    f = paged(plan, 1, 1, 20, fp32=True, max_new=3)          # a token's heads in two tiles
    assert (f["tile_tokens"], f["head_blocks"], f["items"]) == (1, 2, 6)
    assert paged(plan, 1, 8, 5, max_new=4)["tile_tokens"] == 6


@pytest.mark.parametrize("row_bytes", [0, 128, 256, 512])
@pytest.mark.parametrize("batch,kv,group,fp32,max_new,max_len,n_local", [
    (1, 8, 4, False, 1, 98304, 0), (1, 8, 4, False, 1, 16, 0), (48, 8, 8, False, 1, 32768, 0), (65536, 1, 1, False, 1, 1 << 30, 0), (3, 1024, 1, False, 1, 4096, 0),
    (7, 300, 2, True, 1, 4096, 0), (512, 8, 4, True, 8192, 131072, 0), (24, 8, 5, False, 4, 20000, 4096), (2, 1, 64, True, 1 << 20, 1 << 20, 0)])
def test_shares_of_few_rows(plan, batch, kv, group, fp32, max_new, max_len, n_local, row_bytes):
    f = paged(plan, batch, kv, group, fp32, max_tokens=batch * max_new if batch * max_new < 1 << 24 else 1 << 24, max_new=max_new, starts=max_new > 1,
              max_len=max_len, n_local=n_local, row_bytes=row_bytes)
    assert f["rows"] <= 32
    assert 0 <= f["near_shift"] <= 2 and f["set_shift"] <= 3 and kv % (1 << f["set_shift"]) == 0 and f["units"] == 0
    assert f["near_shift"] == 0 or (row_bytes << f["near_shift"] <= 512 and min(group * min(max_new, f["tile_tokens"]), f["rows"]) << f["near_shift"] <= 32)
    row_tiles = batch * -(-max_new // f["tile_tokens"]) * f["head_blocks"]
    charge = -(-max_len // f["key_tile"])
    if n_local:
        charge = min(charge, (n_local + f["tile_tokens"] - 2) // f["key_tile"] + 2)
    # a set only where its parts (of the longest item, if all were as long) can be few enough
    assert f["set_shift"] == 0 or f["target"] << f["set_shift"] <= f["items"] * (16 if f["set_shift"] <= f["near_shift"] and f["items"] * charge >= 128 * f["target"] else 1)
    groups = lambda shift: row_tiles * -(-charge // (1 << (f["group_shift"] - shift)))
    for shift in range(f["set_shift"] + 1):                 # whichever the kernel takes
        sets, most = kv >> shift, f["shares%d" % shift]
        # a counter for every share of a set, a workgroup per compute unit at most, or one for every set
        assert most >= 1 and most * sets <= 1024 and (most == 1 or most * sets <= f["target"])
        # groups of all row tiles are counted in 31 bits; a group has at least a key tile for each of a head's wavefronts
        assert f["group_shift"] >= 3 and groups(shift) + most < 1 << 31
        # the grid and the workspace have room for every share (workgroup i: set (i / 8) % sets, share (i / 8) / sets * 8 + i % 8)
        assert min(f["pieces"] // 8 // sets * 8, f["slots"] // (2 * kv)) >= most
    assert f["group_shift"] == 3 or row_tiles * -(-charge // (1 << (f["group_shift"] - 1 - f["set_shift"]))) + 1024 >= (1 << 31) - 1


@pytest.mark.parametrize("lengths,new,kv,group", [([4099, 2392, 1395, 3337], [4099, 2392, 1395, 3337], 8, 4), ([61440], [2048], 8, 4), ([100000] * 3, [40, 9, 300], 1, 8),
                                                  ([64] * 200, [33] * 200, 2, 4), ([130000, 20], [64, 20], 5, 1), ([1 << 20], [33], 1, 1)])
def test_pieces_of_many_rows_have_room(plan, lengths, new, kv, group):
    f = paged(plan, len(lengths), kv, group, max_tokens=sum(new), max_new=max(new), starts=True, max_len=max(lengths))
    assert f["rows"] == 128
    # what the kernel does with the lengths it finds
    tiles = [-(-t // f["tile_tokens"]) for t in new]
    charge = [max(1, -(-n // f["key_tile"])) for n in lengths]
    total = sum(t * kv * c for t, c in zip(tiles, charge))
    first = max(math.ceil(total * 1.0001 / f["target"]), f["min_tiles"])
    for piece in [first] + [first + (first * k + 7) // 8 for k in range(1, 8)]:   # whichever it takes
        pieces = [-(-c // piece) for c in charge]
        assert sum(t * p for t, p in zip(tiles, pieces)) * kv <= f["pieces"]
        assert sum(t * p for t, p in zip(tiles, pieces) if p > 1) * kv <= f["slots"]
        assert sum(t for t, p in zip(tiles, pieces) if p > 1) * kv <= f["units"]


def test_workgroups_of_the_page_plan(plan):
    go = lambda batch, rows, in_place: plan.plan_workgroups(batch, ctypes.c_long(rows), int(in_place))
    assert [go(64, 64, False), go(64, 4097, True), go(512, 35840, False), go(512, 35840, True), go(2048, 4096, True), go(2049, 10, False), go(2049, 10, True),
            go(5, 1 << 24, False)] == [1, 0, 35, 0, 1, 0, 0, 128]
