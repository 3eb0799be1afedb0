// New keys and values into pools in microscaled 4-bit floating point, and rows of such pools back to bf16.
#include "paged_device.h"

namespace mp {
namespace {

// Sixteen lanes take a row of 128 elements, eight a lane, of the keys and of the values; a quad of lanes has a block of 32.  The scale is
// the least power of two 2^e with max |x| <= 6 * 2^e: with max = 1.m * 2^k, e = k - 2, or k - 1 where 1.m is over 1.5.  Division by it and
// rounding (to nearest, ties to the even code) are one instruction for two elements.  Bound by memory: 16384 tokens of eight heads, 15360 of them with a slot
// (80 MB either way), are stored in 19.4 us, 4.1 TB/s, and read back in 14.3, 5.6 TB/s (four lanes a row, 64 bytes in a lane: 25.6 and 24.1); 64 tokens
// 3.9 and 3.1 us, a launch.

// Magnitudes above 3 * 2^126 as that: their scale is 2^126, of which 4 would be an infinity again.
__device__ inline uint32_t bounded(uint32_t two) {
  constexpr uint32_t kMost = 0x7f40u;
  uint32_t lo = two & 0x7fffu, hi = two >> 16 & 0x7fffu;
  lo = lo > kMost ? kMost : lo;
  hi = hi > kMost ? kMost : hi;
  return (two & 0x80008000u) | hi << 16 | lo;
}

__device__ inline void store_eight(const u32x4& x, uint8_t* row, uint8_t* scale, bool first) {
  uint32_t top = 0;                                        // largest magnitude's bits (in order, NaN above all)
#pragma unroll
  for (int e = 0; e < 4; ++e) top = max(top, max(x[e] & 0x7fffu, x[e] >> 16 & 0x7fffu));
  top = max(top, quad_lane<0xb1>(top));
  top = max(top, quad_lane<0x4e>(top));
  const int exponent = (int)(top >> 7) - 2 + ((top & 0x7fu) > 0x40u);
  uint32_t s = exponent < 0 ? 0 : (uint32_t)exponent, w = 0;
  if (top >= 0x7f80u) {
    s = 255;
  } else {
    const float by = __uint_as_float(s << 23);             // (0 stands for 2^-127)
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x[0])), by, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x[1])), by, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x[2])), by, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, bounded(x[3])), by, 3);
  }
  *reinterpret_cast<uint32_t*>(row) = w;
  if (first) *scale = (uint8_t)s;
}

// f(row's place among the tokens' rows, where its keys' and values' elements lie in the pools) for the rows that have a slot; two at a time.
struct Places {
  int64_t k_row, v_row, k, v;
  bool there;
};
__device__ inline Places places_of(const PageMxfp4Args& a, int64_t r, int64_t rows, int l) {
  Places p{0, 0, 0, 0, false};
  if (r >= rows) return p;
  const int64_t t = r / a.heads;
  const int h = (int)(r - t * a.heads);
  const int64_t slot = a.slots[t], page = slot >> a.page_shift, at = slot & ((1 << a.page_shift) - 1);
  p.there = slot >= 0 && slot < a.n_slots;
  p.k_row = t * a.kn_t + h * a.kn_h + 8 * l;
  p.v_row = t * a.vn_t + h * a.vn_h + 8 * l;
  p.k = page * a.k_page + at * a.k_key + h * a.k_head + 8 * l;
  p.v = page * a.v_page + at * a.v_key + h * a.v_head + 8 * l;
  return p;
}

constexpr int kAtOnce = 2;                                // rows of a group of sixteen lanes
template <bool APPEND>
__global__ __launch_bounds__(256) void page_mxfp4_kernel(const PageMxfp4Args a) {
  const int64_t rows = a.tokens * a.heads, stride = (int64_t)gridDim.x * 16 * kAtOnce;
  const int l = threadIdx.x & 15;
  for (int64_t r = (int64_t)blockIdx.x * 16 * kAtOnce + (threadIdx.x >> 4); r < rows; r += stride) {
    Places p[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) p[i] = places_of(a, r + 16 * i, rows, l);
    if constexpr (APPEND) {
      u32x4 k[kAtOnce], v[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        k[i] = v[i] = u32x4{0, 0, 0, 0};
        if (p[i].there) {
          k[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.k_rows) + p[i].k_row));
          v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.v_rows) + p[i].v_row));
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (!p[i].there) continue;                         // (the same for a row's lanes)
        store_eight(k[i], a.k_pages + (p[i].k >> 1), a.k_block + (p[i].k >> 5), (l & 3) == 0);
        store_eight(v[i], a.v_pages + (p[i].v >> 1), a.v_block + (p[i].v >> 5), (l & 3) == 0);
      }
    } else {
      uint32_t k[kAtOnce], v[kAtOnce], ks[kAtOnce], vs[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        k[i] = v[i] = ks[i] = vs[i] = 0;
        if (p[i].there) {
          k[i] = *reinterpret_cast<const uint32_t*>(a.k_pages + (p[i].k >> 1));
          v[i] = *reinterpret_cast<const uint32_t*>(a.v_pages + (p[i].v >> 1));
          ks[i] = a.k_block[p[i].k >> 5];
          vs[i] = a.v_block[p[i].v >> 5];
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (!p[i].there) continue;
        __builtin_nontemporal_store(e2m1_to_bf16(k[i], ks[i] << 23), reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(a.k_rows) + p[i].k_row));
        __builtin_nontemporal_store(e2m1_to_bf16(v[i], vs[i] << 23), reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(a.v_rows) + p[i].v_row));
      }
    }
  }
}

dim3 grid_of(const PageMxfp4Args& a) {
  const int64_t blocks = (a.tokens * a.heads + 16 * kAtOnce - 1) / (16 * kAtOnce), most = 64 * kNumCU;
  return dim3((unsigned)(blocks < most ? blocks : most));
}

}  // namespace

hipError_t launch_page_append_mxfp4(const PageMxfp4Args& a, hipStream_t s) {
  page_mxfp4_kernel<true><<<grid_of(a), 256, 0, s>>>(a);
  return hipGetLastError();
}
hipError_t launch_page_read_mxfp4(const PageMxfp4Args& a, hipStream_t s) {
  page_mxfp4_kernel<false><<<grid_of(a), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mp
