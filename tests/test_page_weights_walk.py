"""How the form for many rows of the accounts walks over query rows: a lane's 32-bit offset from a pointer that goes along, compiled on its own."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# The kernel's steps from row `begin` on, lane offsets as it forms them.  0, or 1 + the step at which a row is not where it should be or an offset leaves 31 bits.
SHIM = """
#include "launch_plan.h"
extern "C" long walk(long q_t, long q_h, int group, int heads, int begin, int step, long rows, long* farthest) {
  const int dt = step / group, dh = step - dt * group, t0 = begin / group;
  const long wrap = q_t - group * q_h;
  int first_head = begin - t0 * group, head[32];
  long at = t0 * q_t, lse_at = (long)t0 * heads, from[32], lse_from[32], n = 0;
  for (int j = 0; j < 32; ++j) {
    const int t = (begin + j) / group;
    head[j] = begin + j - t * group;
    from[j] = (t - t0) * q_t + head[j] * q_h;
    lse_from[j] = (t - t0) * heads + head[j];
  }
  *farthest = 0;
  for (long r = begin; r < rows; r += step, ++n) {
    for (int j = 0; j < 32; ++j) {
      const long t = (r + j) / group, h = (r + j) % group, far = from[j] < 0 ? -from[j] : from[j];
      if (far > *farthest) *farthest = far;
      if (at + from[j] != t * q_t + h * q_h || lse_at + lse_from[j] != t * heads + h) return 1 + n;
      if (far + 496 > 2147483647L || lse_from[j] != (int)lse_from[j]) return 1 + n;
    }
    const bool past = mp::next_head(first_head, dh, group);
    at += dt * q_t + dh * q_h + (past ? wrap : 0);
    lse_at += (long)dt * heads + dh + (past ? heads - group : 0);
    for (int j = 0; j < 32; ++j) {
      const bool own = mp::next_head(head[j], dh, group);
      from[j] += mp::offset_step(own, past, (int)wrap);
      lse_from[j] += mp::offset_step(own, past, heads - group);
    }
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("walk")
    (tmp / "shim.cpp").write_text(SHIM)
    so = str(tmp / "shim.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2410_16179_amd", "csrc"), str(tmp / "shim.cpp"), "-o", so], check=True)
    f = ctypes.CDLL(so).walk
    f.restype, f.argtypes = ctypes.c_long, [ctypes.c_long] * 2 + [ctypes.c_int] * 4 + [ctypes.c_long, ctypes.POINTER(ctypes.c_long)]

    def of(q_t, q_h, group, kv_heads, begin, step, rows):
        far = ctypes.c_long()
        return f(q_t, q_h, group, group * kv_heads, begin, step, rows, far), far.value
    return of


LARGEST = 4 << 22                                             # bytes of the largest stride, float32


@pytest.mark.parametrize("step", [32, 64, 128])
@pytest.mark.parametrize("group", list(range(1, 65)))
def test_every_row_is_found_within_31_bits(walk, group, step):
    for q_t, q_h in ((group * 8 * 256, 256), (LARGEST, 256), (LARGEST, LARGEST), (512, LARGEST), (0, 512), (LARGEST, 0)):
        for begin in (0, 16, 48, 16 * group, 96 + 16 * (group // 2)):
            found, far = walk(q_t, q_h, group, 8, begin, step, 20000)
            assert found == 0, (q_t, q_h, begin, far)


def test_a_long_prompt_of_rows_that_lie_far_apart(walk):
    # (an offset from a pointer that takes no part in the wraps passes 2^31 behind some hundred tokens)
    assert walk(2 << 22, 256, 43, 2, 0, 128, 1000 * 43)[0] == 0
    assert walk(4 << 22, 512, 43, 2, 0, 128, 520 * 43)[0] == 0
    for group, kv_heads in ((3, 8), (5, 8), (40, 8), (63, 1024)):
        found, far = walk(group * kv_heads * 256, 256, group, kv_heads, 0, 128, 1 << 22)
        assert found == 0 and far < 1 << 26
