// New keys and values into pools in microscaled 4-bit floating point, and rows of such pools back to bf16.
#include "paged_device.h"

namespace mp {
namespace {

// Four lanes take a row, a block of 32 elements each, of the keys and of the values: 64 bytes in, sixteen out, and a byte of scale.  The scale is
// the least power of two 2^e with max |x| <= 6 * 2^e: with max = 1.m * 2^k, e = k - 2, or k - 1 where 1.m is over 1.5.  Division by it and
// rounding (to nearest, ties to the even code) are one instruction for two elements.  Bound by memory.
struct Row {
  u32x4 w[4];
};

// Magnitudes above 3 * 2^126 as that: their scale is 2^126, of which 4 would be an infinity again.
__device__ inline uint32_t bounded(uint32_t two) {
  constexpr uint32_t kMost = 0x7f40u;
  uint32_t lo = two & 0x7fffu, hi = two >> 16 & 0x7fffu;
  lo = lo > kMost ? kMost : lo;
  hi = hi > kMost ? kMost : hi;
  return (two & 0x80008000u) | hi << 16 | lo;
}

__device__ inline void store_block(const Row& x, uint8_t* row, uint8_t* scale) {
  uint32_t top = 0;                                        // largest magnitude's bits (in order, NaN above all)
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = x.w[i][e] & 0x7fffu, hi = x.w[i][e] >> 16 & 0x7fffu;
      top = max(top, max(lo, hi));
    }
  const int exponent = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x40u);
  uint32_t s = exponent < 0 ? 0 : (uint32_t)exponent;
  u32x4 codes = {0, 0, 0, 0};
  if (top >= 0x7f80u) {
    s = 255;
  } else {
    const float by = __uint_as_float(s << 23);             // (0 stands for 2^-127)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w = 0;
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x.w[i][0])), by, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x.w[i][1])), by, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x.w[i][2])), by, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x.w[i][3])), by, 3);
      codes[i] = w;
    }
  }
  *reinterpret_cast<u32x4*>(row) = codes;
  *scale = (uint8_t)s;
}

__device__ inline void load_row(const void* rows, int64_t element, Row& x) {
  const u32x4* from = reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(rows) + element);
#pragma unroll
  for (int i = 0; i < 4; ++i) x.w[i] = __builtin_nontemporal_load(from + i);
}

__global__ __launch_bounds__(256) void page_append_mxfp4_kernel(const PageMxfp4Args a) {
  const int64_t rows = a.tokens * a.heads, stride = (int64_t)gridDim.x * 64;
  const int l = threadIdx.x & 3;
  for (int64_t r = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2); r < rows; r += stride) {
    const int64_t t = r / a.heads;
    const int h = (int)(r - t * a.heads);
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) continue;
    Row k, v;
    load_row(a.k_rows, t * a.kn_t + h * a.kn_h + 32 * l, k);
    load_row(a.v_rows, t * a.vn_t + h * a.vn_h + 32 * l, v);
    const int64_t page = slot >> a.page_shift, at = slot & ((1 << a.page_shift) - 1);
    const int64_t ke = page * a.k_page + at * a.k_key + h * a.k_head + 32 * l, ve = page * a.v_page + at * a.v_key + h * a.v_head + 32 * l;
    store_block(k, a.k_pages + (ke >> 1), a.k_block + (ke >> 5));
    store_block(v, a.v_pages + (ve >> 1), a.v_block + (ve >> 5));
  }
}

__device__ inline void read_block(const uint8_t* row, const uint8_t* scale, void* rows, int64_t element) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(row);
  const uint32_t s = (uint32_t)*scale << 23;
  u32x4* to = reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(rows) + element);
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = e2m1_to_bf16(w[i], s);
}

__global__ __launch_bounds__(256) void page_read_mxfp4_kernel(const PageMxfp4Args a) {
  const int64_t rows = a.tokens * a.heads, stride = (int64_t)gridDim.x * 64;
  const int l = threadIdx.x & 3;
  for (int64_t r = (int64_t)blockIdx.x * 64 + (threadIdx.x >> 2); r < rows; r += stride) {
    const int64_t t = r / a.heads;
    const int h = (int)(r - t * a.heads);
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) continue;
    const int64_t page = slot >> a.page_shift, at = slot & ((1 << a.page_shift) - 1);
    const int64_t ke = page * a.k_page + at * a.k_key + h * a.k_head + 32 * l, ve = page * a.v_page + at * a.v_key + h * a.v_head + 32 * l;
    read_block(a.k_pages + (ke >> 1), a.k_block + (ke >> 5), a.k_rows, t * a.kn_t + h * a.kn_h + 32 * l);
    read_block(a.v_pages + (ve >> 1), a.v_block + (ve >> 5), a.v_rows, t * a.vn_t + h * a.vn_h + 32 * l);
  }
}

dim3 grid_of(const PageMxfp4Args& a) {
  const int64_t blocks = (a.tokens * a.heads + 63) / 64, most = 64 * kNumCU;
  return dim3((unsigned)(blocks < most ? blocks : most));
}

}  // namespace

hipError_t launch_page_append_mxfp4(const PageMxfp4Args& a, hipStream_t s) {
  page_append_mxfp4_kernel<<<grid_of(a), 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_page_read_mxfp4(const PageMxfp4Args& a, hipStream_t s) {
  page_read_mxfp4_kernel<<<grid_of(a), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mp
