// New keys and values into their slots of the paged pools.
#include "paged_common.h"

#include <type_traits>

namespace mp {
namespace {

// Sixteen lanes take a row of 128 elements, eight a lane, of the keys and of the values: each lane reads its 16
// bytes (bf16) of both and stores what they become.  Bound by memory: 2 rows in, 2 rows out.  16384 tokens of eight heads, 15360 of them with a slot,
// in graph replay: into e4m3 pools (94.5 MB) 23 us, 4.1 TB/s, bf16 (126 MB) 24, 5.2 TB/s, float32 (252 MB) 59, 4.3 TB/s (a large copy 4.9); called one
// behind the other e4m3 takes 21.5.  Rows without a slot are read all the same: their loads are requested beside the slot's.  64 tokens 2.5 us, a launch.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int ET>
struct Eight;                                             // eight elements of a pool, as stored
template <>
struct Eight<kBF16> { u32x4 w; };
template <>
struct Eight<kFP32> { u32x4 w, w2; };
template <>
struct Eight<kFP8> { u32x2 w; };

__device__ inline float to_e4m3_range(float x) {          // (comparisons are false of a NaN: it stays)
  x = x > 448.f ? 448.f : x;
  return x < -448.f ? -448.f : x;
}

// x / scale as correctly rounded as a division gives it, from the reciprocal: the product's remainder is exact (a fused
// multiply-add), and what it lacks is added.  Beyond 512 the product stands (it is clamped, an infinity and a NaN among them); the sign is the
// product's (a zero's would be lost).  A quarter of a division's instructions, which were what e4m3 pools waited for:
// that case, graph replay, 28.3 us with divisions, 24.2 so (then with ordinary stores).
__device__ inline float quotient(float x, float scale, float inverse) {
  const float q = x * inverse;
  const float r = __builtin_copysignf(fmaf(fmaf(-q, scale, x), inverse, q), q);
  return fabsf(q) < 512.f ? r : q;
}

template <int ET>
__device__ inline Eight<ET> convert(const Frag& f, float scale) {
  Eight<ET> r;
  if constexpr (ET == kFP8) {
    float v[8];
    frag_to_float<kBF16>(f, v);
    if (fabsf(scale) > 0x1p-100f && fabsf(scale) < 0x1p100f) {
      const float inverse = 1.f / scale;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_e4m3_range(quotient(v[e], scale, inverse));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = to_e4m3_range(v[e] / scale);
    }
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    r.w = u32x2{(uint32_t)lo, (uint32_t)hi};
  } else if constexpr (ET == kFP32) {
    r.w = __builtin_bit_cast(u32x4, f.a);
    r.w2 = __builtin_bit_cast(u32x4, f.b);
  } else {
    r.w = __builtin_bit_cast(u32x4, f.a);
  }
  return r;
}
// (not kept in the caches: a step reads what it stored long after)
template <int ET>
__device__ inline void store(const Eight<ET>& r, char* to) {
  __builtin_nontemporal_store(r.w, reinterpret_cast<std::remove_const_t<decltype(r.w)>*>(to));
  if constexpr (ET == kFP32) __builtin_nontemporal_store(r.w2, reinterpret_cast<u32x4*>(to + 16));
}

template <int ET>
__global__ __launch_bounds__(256) void page_append_kernel(const PageAppendArgs a) {
  constexpr int kElem = ET == kFP32 ? 4 : (ET == kFP8 ? 1 : 2);
  constexpr int kIn = ET == kFP32 ? kFP32 : kBF16;
  const int64_t rows = a.tokens * a.heads, stride = (int64_t)gridDim.x * 16;
  const int l = threadIdx.x & 15;
  for (int64_t r = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); r < rows; r += stride) {
    const int64_t t = r / a.heads;
    const int h = (int)(r - t * a.heads);
    const int64_t slot = a.slots[t];
    Frag k, v;
    frag_load<kIn>(a.k_new, t * a.kn_t + h * a.kn_h + l * 8, k);
    frag_load<kIn>(a.v_new, t * a.vn_t + h * a.vn_h + l * 8, v);
    if (slot < 0 || slot >= a.n_slots) continue;
    const int64_t page = slot >> a.page_shift, at = slot & ((1 << a.page_shift) - 1);
    char* kp = reinterpret_cast<char*>(a.k_pages) + (page * a.k_page + at * a.k_key + h * a.k_head + l * 8) * kElem;
    char* vp = reinterpret_cast<char*>(a.v_pages) + (page * a.v_page + at * a.v_key + h * a.v_head + l * 8) * kElem;
    store<ET>(convert<ET>(k, a.k_scale ? a.k_scale[h] : 1.f), kp);
    store<ET>(convert<ET>(v, a.v_scale ? a.v_scale[h] : 1.f), vp);
  }
}

}  // namespace

hipError_t launch_page_append(const PageAppendArgs& a, hipStream_t s) {
  const int64_t blocks = (a.tokens * a.heads + 15) / 16, most = 64 * kNumCU;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  if (a.is_fp32) page_append_kernel<kFP32><<<grid, 256, 0, s>>>(a);
  else if (a.kv_fp8) page_append_kernel<kFP8><<<grid, 256, 0, s>>>(a);
  else page_append_kernel<kBF16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mp
