"""The rules of csrc/launch_plan.h for pools in four bits, accounts, the keys that stay and eviction, compiled on their own."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = """
#include "launch_plan.h"
extern "C" {
void paged(int batch, int kv, int group, long max_tokens, int max_new, int starts, long max_len, int n_local, int row_bytes, long* got) {
  const mp::PagedForm f = mp::paged_form(batch, kv, group, false, max_tokens, max_new, starts, max_len, 0, n_local, row_bytes, true);
  const long all[] = {f.rows, f.key_tile, f.tile_tokens, f.head_blocks, f.target, f.near_shift, f.set_shift, f.group_shift, f.shares[0], f.shares[1], f.shares[2], f.shares[3],
                      f.items, f.pieces, f.slots};
  for (int i = 0; i < 15; ++i) got[i] = all[i];
}
void weights(int batch, int kv, int group, int fp32, int bits, int max_new, long max_len, long* got) {
  const mp::WeightsForm f = mp::weights_form(batch, kv, group, fp32, bits, max_new, max_len);
  got[0] = f.many; got[1] = f.rows; got[2] = f.heads; got[3] = f.tiles; got[4] = f.workgroups; got[5] = mp::weights_fit(f);
}
int parts(long rows, long max_len) { return mp::keep_parts(rows, max_len); }
int slice(int row, long units) { return mp::evict_slice(row, units); }
}
"""
PAGED = ("rows", "key_tile", "tile_tokens", "head_blocks", "target", "near_shift", "set_shift", "group_shift", "shares0", "shares1", "shares2", "shares3", "items",
         "pieces", "slots")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("plan")
    (tmp / "shim.cpp").write_text(SHIM)
    so = str(tmp / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2410_16179_amd", "csrc"), str(tmp / "shim.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


@pytest.mark.parametrize("row_bytes", [0, 64])
@pytest.mark.parametrize("batch,kv,group,max_new,max_len,n_local", [
    (1, 8, 4, 1, 98304, 0), (1, 8, 4, 1, 16, 0), (48, 8, 8, 1, 30016, 0), (65536, 1, 1, 1, 1 << 30, 0), (3, 1024, 1, 1, 4096, 0), (24, 8, 5, 4, 20000, 4096),
    (64, 32, 1, 1, 2000, 0), (16, 8, 4, 1, 65536, 0), (7, 300, 2, 1, 4096, 0)])
def test_shares_of_few_rows(plan, batch, kv, group, max_new, max_len, n_local, row_bytes):
    got = (ctypes.c_long * 15)()
    plan.paged(batch, kv, group, ctypes.c_long(batch * max_new), max_new, int(max_new > 1), ctypes.c_long(max_len), n_local, row_bytes, got)
    f = dict(zip(PAGED, got))
    assert f["key_tile"] == 64 and f["rows"] <= 32
    assert f["set_shift"] <= 3 and kv % (1 << f["set_shift"]) == 0 and row_bytes << f["near_shift"] <= 512
    row_tiles = batch * -(-max_new // f["tile_tokens"]) * f["head_blocks"]
    charge = -(-max_len // 64)
    if n_local:
        charge = min(charge, (n_local + f["tile_tokens"] - 2) // 64 + 2)
    for shift in range(f["set_shift"] + 1):
        sets, most = kv >> shift, f["shares%d" % shift]
        # counters, a workgroup per compute unit, groups in 31 bits, room for every share and its partials
        assert most >= 1 and most * sets <= 1024 and (most == 1 or most * sets <= f["target"])
        assert row_tiles * -(-charge // (1 << (f["group_shift"] - shift))) + most < 1 << 31
        assert min(f["pieces"] // 8 // sets * 8, f["slots"] // (2 * kv)) >= most


def weights(plan, batch, kv, group, max_new, max_len, fp32=False, bits=16):
    got = (ctypes.c_long * 6)()
    plan.weights(batch, kv, group, int(fp32), bits, max_new, ctypes.c_long(max_len), got)
    return dict(zip(("many", "rows", "heads", "tiles", "workgroups", "fit"), got))


@pytest.mark.parametrize("bits", [4, 8, 16, 32])
@pytest.mark.parametrize("group,max_new", [(1, 1), (16, 1), (17, 1), (4, 8), (5, 7), (64, 1), (4, 20), (64, 2), (43, 3), (64, 64), (1, 1 << 24)])
def test_rows_of_the_accounts_forms(plan, bits, group, max_new):
    for kv in (1, 2, 3, 8, 12, 1024):
        for batch, max_len in ((1, 16), (1, 98304), (64, 4096)):
            f = weights(plan, batch, kv, group, max_new, max_len, fp32=bits == 32, bits=min(bits, 16))
            rows = group * max_new
            if f["many"]:
                assert rows > (16 if bits == 32 else 128) and f["heads"] in (1, 2, 4) and (f["heads"] == 1 or 32 * f["heads"] <= rows)
                tile, per = (32 if bits == 32 else 64) * 4 // f["heads"], kv
            else:
                # a wavefront has all rows, and its workgroup whole sets of KV heads
                assert rows <= f["rows"] <= (16 if bits == 32 else 128) and kv % f["heads"] == 0 and f["heads"] in (1, 2, 4, 8)
                tile, per = (16 if bits == 32 else 32 if bits == 16 or f["rows"] > 16 else 64), kv
            assert f["tiles"] == -(-max_len // tile) * batch * per
            assert 1 <= f["workgroups"] <= 1 << 14 and f["fit"]


def test_more_tiles_than_are_counted(plan):
    assert not weights(plan, 65536, 64, 1, 1, 1 << 24)["fit"]
    assert weights(plan, 64, 8, 4, 1, 1 << 26)["fit"]


def test_workgroups_to_a_request(plan):
    parts = lambda rows, n: plan.parts(ctypes.c_long(rows), ctypes.c_long(n))
    assert [parts(8, 24576), parts(8, 24577), parts(8, 98304), parts(33, 98304), parts(1, 1 << 20), parts(1, 16 * 65280), parts(32, 200000)] == [1, 4, 12, 1, 1, 16, 16]
    for n in range(24577, 16 * 65280, 7777):                  # a part's counts have 16 bits
        p = parts(1, n)
        assert 4 <= p <= 16 and (-(-n // p) + 255) // 256 * 256 <= 65535


def test_slices(plan):
    for row in (64, 128, 256, 512):
        for units in (1, 8, 16, 32, 64, 128, 1000):
            s = plan.slice(row, ctypes.c_long(units))
            assert 32 <= s <= row and row % s == 0 and s % 16 == 0
            assert s == row or 2 * units * (row // (2 * s)) < 256
