// Pieces shared by the kernels of paged attention: matrix products, conversions, loads of pool rows.
#pragma once
#include "paged_common.h"

namespace mp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef const int __attribute__((address_space(4))) * const_i32_ptr;

constexpr int kPartialRow = kPartialStride;   // floats of a row's partial: 128 outputs, maximum, sum, pad

// Eight e4m3 bytes as eight bf16 (exact), two per instruction.
__device__ inline u32x4 e4m3_to_bf16(u32x2 w) {
  u32x4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, true));
  return r;
}

// Eight e2m1 elements, four bytes, times 2^(scale - 127) as eight bf16, two per instruction: exact but where bf16 overflows (to an
// infinity) or ends (below 2^-133); scale 255 gives NaN.  scale: the e8m0 byte in bits 23 .. 30 (the instruction looks at no others).
__device__ inline u32x4 e2m1_to_bf16(uint32_t w, uint32_t scale) {
  const float s = __uint_as_float(scale);
  u32x4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  return r;
}
// What has to be rotated right to bring byte `i` of a word to bits 23 .. 30.
__device__ inline int to_scale(int i) { return (8 * i + 9) & 31; }
__device__ inline uint32_t rotate_right(uint32_t w, int by) { return __builtin_amdgcn_alignbit(w, w, by); }

// Bytes of so many elements of a pool (a multiple of two of kFP4).
template <int ET>
__device__ inline int64_t pool_bytes(int64_t elements) {
  return ET == kFP4 ? elements >> 1 : elements * (ET == kFP32 ? 4 : (ET == kFP8 ? 1 : 2));
}

__device__ inline uint32_t pack_bf16(float lo, float hi) {
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ inline f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Loads through a buffer descriptor, not kept in the caches (nt): a decoding step reads a row once.  Where a request has several row tiles (more new tokens
// than 16 or 32 rows hold: float32 prompts above all) each of them reads the rows again, in this way too.
constexpr int kBufferWord3 = 0x00020000;
constexpr int kNonTemporal = 2;
__device__ inline void load_once(__amdgpu_buffer_rsrc_t rows, uint32_t at, u32x4& to) {
  to = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at, 0, kNonTemporal));
}
__device__ inline void load_once(__amdgpu_buffer_rsrc_t rows, uint32_t at, u32x2& to) {
  to = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, at, 0, kNonTemporal));
}
__device__ inline uint32_t load_byte(__amdgpu_buffer_rsrc_t rows, uint32_t at) { return __builtin_amdgcn_raw_buffer_load_b8(rows, at, 0, 0); }
// The same, kept: workgroups of other row tiles read the row too.
__device__ inline void load_shared(__amdgpu_buffer_rsrc_t rows, uint32_t at, u32x4& to) {
  to = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at, 0, 0));
}
__device__ inline void load_shared(__amdgpu_buffer_rsrc_t rows, uint32_t at, u32x2& to) {
  to = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, at, 0, 0));
}
__device__ inline void load_shared(__amdgpu_buffer_rsrc_t rows, uint32_t at, uint32_t& to) {
  to = __builtin_amdgcn_raw_buffer_load_b32(rows, at, 0, 0);
}

// The lanes' 16 bytes one behind the other from `to` on (the same for the wavefront); there behind stored().
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t rows, uint32_t at, char* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, 0);
}

// Partial results that another workgroup joins within the same launch.  Workgroups may sit on different XCDs, whose L2s do not see one
// another's lines.  A release and an acquire at agent scope would write back and drop whole L2s, in every workgroup
// (the step of one user at 96k took 220 us for 81); instead the values themselves go past the L2s, as relaxed atomics
// of agent scope.  stored() waits until what this wavefront has under way has arrived.
__device__ inline void store_through(float* to, float x, float y) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(to), (uint64_t)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline f32x2 load_through(const float* from) {
  const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return f32x2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}
__device__ inline void stored() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Between what a wavefront's lanes write to its own part of LDS and what others of its lanes read there: the unit takes a wavefront's
// accesses in their order, so only the compiler has to keep it.
__device__ inline void in_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// w without infinities and NaN: a float32, or two bf16.
template <bool F32>
__device__ inline uint32_t finite_part(uint32_t w) {
  if constexpr (F32) return (w & 0x7f800000u) == 0x7f800000u ? 0u : w;
  return ((w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u);
}
template <bool F32>
__device__ inline u32x4 finite_part(u32x4 w) {
  return u32x4{finite_part<F32>(w.x), finite_part<F32>(w.y), finite_part<F32>(w.z), finite_part<F32>(w.w)};
}

// Keys are loaded with neighbouring lanes on neighbouring addresses - a quad of lanes reads 64 bytes of one key - and then
// change lanes inside the quad, where an MFMA operand has a key per lane: with a key per lane from the start a load
// meets 64 addresses apart from each other, which the L1 takes one by one (58 % of its time in e4m3 decoding).
template <int CTRL>
__device__ inline uint32_t quad_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
// (every lane takes part in an exchange: it stands before the choice, not inside it)
// r[i] of lane j of a quad <-> r[j] of lane i.
__device__ inline void transpose_quads(u32x4& r0, u32x4& r1, u32x4& r2, u32x4& r3, bool odd, bool upper) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x0 = quad_lane<0xb1>(r0[e]), x1 = quad_lane<0xb1>(r1[e]), x2 = quad_lane<0xb1>(r2[e]), x3 = quad_lane<0xb1>(r3[e]);   // lane ^ 1
    const uint32_t a0 = odd ? x1 : r0[e], a1 = odd ? r1[e] : x0, a2 = odd ? x3 : r2[e], a3 = odd ? r3[e] : x2;
    const uint32_t y0 = quad_lane<0x4e>(a0), y1 = quad_lane<0x4e>(a1), y2 = quad_lane<0x4e>(a2), y3 = quad_lane<0x4e>(a3);               // lane ^ 2
    r0[e] = upper ? y2 : a0;
    r1[e] = upper ? y3 : a1;
    r2[e] = upper ? a2 : y0;
    r3[e] = upper ? a3 : y1;
  }
}
// Lane j of a quad has half j % 2 of keys j / 2 (r0) and 2 + j / 2 (r1) -> both halves of key j.
__device__ inline void join_halves(u32x4& r0, u32x4& r1, bool upper) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t x0 = quad_lane<0x88>(r0[e]), x1 = quad_lane<0x88>(r1[e]);                             // lanes 0, 2, 0, 2
    const uint32_t y0 = quad_lane<0xdd>(r0[e]), y1 = quad_lane<0xdd>(r1[e]);                             // lanes 1, 3, 1, 3
    r0[e] = upper ? x1 : x0;
    r1[e] = upper ? y1 : y0;
  }
}

// The pages of a tile, one for every 16 keys: ids as the table has them.
template <int KT>
struct TilePages {
  int id[KT / 16];
};

// Descriptor of 16 keys' rows of a pool, from key `at` of page `id` on, `valid` of which are there: the others lie beyond the
// descriptor's end and read as zeros, without an access.  Strides in bytes.
__device__ inline __amdgpu_buffer_rsrc_t rows16(const char* pool, int64_t page_stride, uint32_t key_stride, int id, int at, int valid) {
  const char* base = pool + (valid ? id : 0) * page_stride + (uint32_t)at * key_stride;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, valid * key_stride, kBufferWord3);
}

}  // namespace mp
