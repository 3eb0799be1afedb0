// Exact attention over a paged key-value cache: the form for many rows per KV head (prompts, chunks of prompts).
#include "paged_device.h"

#include <type_traits>

namespace mp {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int KT = kPagedManyKeys, R = kPagedManyRows;
constexpr int kTileBytes = KT * kHeadDim * 2;             // a tile of keys or values as bf16

__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Four values of this lane's column, from a block of four rows by sixteen columns that sixteen lanes point at.
__device__ inline u32x2 read_transposed(const char* lds) {
  typedef i16x4 __attribute__((address_space(3))) * lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds)));
}

// Four wavefronts share tiles of 64 keys in LDS (two buffers); each has 32 query rows.  As in the form for few rows
// both products are formed transposed, here with the 32 x 32 x 16 MFMA: S^T = K Q^T has keys along an
// accumulator's registers and a query row in a lane (and the lane 32 further on), so maximum, weights and sum need
// no exchange but one between two lanes, and the weights are the B operand of O^T = V^T P^T as they are.
// A operands come from LDS: K rows by 16-byte reads, V^T by the transposing read, four keys of a column at a
// time.  16-byte chunks of a row are stored at places that depend on the key (chunk ^ key % 16 of K, and
// chunk ^ 4 (key % 4) of V), so that the lanes of a read meet different banks.
// Weights are rounded to bf16 (half a step is 2^-8 of a weight): a second product with what the rounding left
// would cost half as much matrix work again, and the output is rounded to bf16 anyway.
template <int ET>
__global__ __launch_bounds__(256, 2) void paged_many_rows_kernel(const PagedArgs a) {
  constexpr int kElem = ET == kFP8 ? 1 : 2;
  typedef typename std::conditional<ET == kFP8, u32x2, u32x4>::type Raw;
  __shared__ __align__(16) char lds[2][2][kTileBytes];     // [buffer][keys, values]

  PagedPiece pc;
  if (!paged_locate<KT, kPieces>(a, blockIdx.x, pc)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 31, u = lane >> 5;
  const int len = pc.r.len, tokens = pc.r.tokens;
  const int tt = pc.tile / a.head_blocks, hb = pc.tile - tt * a.head_blocks;
  const int first = tt * a.tile_tokens, last = min(first + a.tile_tokens, tokens) - 1;
  const int heads = min(a.G - hb * R, R);
  const int rows = a.head_blocks > 1 ? heads : (last - first + 1) * a.G;
  const PagedSpan span = paged_span<KT>(a, len, tokens, first, last);
  int t_begin, t_end;
  paged_piece_range(span.count, pc.piece, pc.pieces, t_begin, t_end);

  auto token_of = [&](int row) { return a.head_blocks > 1 ? 0 : row / a.G; };
  const int row = 32 * wave + c, t = token_of(row), head = a.head_blocks > 1 ? hb * R + row : row - t * a.G;
  const bool real = row < rows;
  const int hi = real ? len - tokens + first + t : -1, lo = a.n_local > 0 ? hi - a.n_local + 1 : 0;
  // the wavefront's rows: what all of them attend is [max_lo, min_hi], what one of them attends ends at wave_hi
  const bool busy = 32 * wave < rows;
  const int t0 = token_of(32 * wave), t1 = token_of(min(32 * wave + 31, rows - 1));
  const int min_hi = len - tokens + first + t0, wave_hi = busy ? len - tokens + first + t1 : -1;
  const int max_lo = a.n_local > 0 ? wave_hi - a.n_local + 1 : 0;
  const int end = len - tokens + last + 1;
  const int any_lo = a.n_local > 0 ? len - tokens + first - a.n_local + 1 : 0;
  // a negative scale goes to the queries, so that the largest score is the largest product
  const float signed_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[pc.g] : 1.f), to_log2 = fabsf(signed_log2);
  const uint32_t flip = signed_log2 < 0.f ? 0x80008000u : 0u;

  u32x4 q[8];
  {
    const int64_t at = (int64_t)(pc.r.row + first + t) * a.q_t + (int64_t)(pc.g * a.G + head) * a.q_h + 8 * u;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      q[s] = u32x4{0, 0, 0, 0};
      if (real) q[s] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + at + 16 * s) ^ flip;
    }
  }

  const const_i32_ptr table = (const_i32_ptr)(a.table + (int64_t)pc.b * a.max_pages);
  const char* kbase = reinterpret_cast<const char*>(a.k) + (int64_t)pc.g * a.k_head * kElem;
  const char* vbase = reinterpret_cast<const char*>(a.v) + (int64_t)pc.g * a.v_head * kElem;
  const int page_mask = (1 << a.page_shift) - 1;
  const uint32_t k_key = (uint32_t)a.k_key * kElem, v_key = (uint32_t)a.v_key * kElem;
  // staging: sixteen lanes take a row, the workgroup sixteen rows at a time
  const int srow = threadIdx.x >> 4, chunk = threadIdx.x & 15;
  const uint32_t k_from = srow * k_key + 8 * chunk * kElem, v_from = srow * v_key + 8 * chunk * kElem;
  const int k_to = srow * 256 + ((chunk ^ srow) << 4), v_to = srow * 256 + ((chunk ^ (srow & 3) << 2) << 4);
  // reading
  const int k_at = c * 256, k_swap = (u ^ (c & 15)) << 4;
  const int i16 = lane & 15, quad = i16 >> 2;
  const int v_at = (4 * u + quad) * 256 + (2 * (lane >> 4 & 1) + (i16 >> 1 & 1)) * 16 + (i16 & 1) * 8;

  auto tile_key = [&](int v) { return (v < span.sink ? v : v + span.skip) * KT; };
  auto page_ok = [&](int id) { return (uint32_t)id < (uint32_t)a.n_pages; };
  auto tile_pages = [&](int v, TilePages<KT>& p) {
    const int key0 = tile_key(v);
#pragma unroll
    for (int h = 0; h < KT / 16; ++h) {
      const int at = (key0 + 16 * h) >> a.page_shift;
      p.id[h] = table[at < a.max_pages ? at : a.max_pages - 1];
    }
  };
  Raw kr[KT / 16], vr[KT / 16];
  auto fetch = [&](int v, const TilePages<KT>& p) {
    const int key0 = tile_key(v);
#pragma unroll
    for (int h = 0; h < KT / 16; ++h) {
      const int at = key0 + 16 * h, valid = page_ok(p.id[h]) ? min(max(end - at, 0), 16) : 0;
      load_shared(rows16(kbase, a.k_page * kElem, k_key, p.id[h], at & page_mask, valid), k_from, kr[h]);
      load_shared(rows16(vbase, a.v_page * kElem, v_key, p.id[h], at & page_mask, valid), v_from, vr[h]);
    }
  };
  auto put = [&](int buf, int key0, auto careful) {
#pragma unroll
    for (int h = 0; h < KT / 16; ++h) {
      u32x4 k, v;
      if constexpr (ET == kFP8) { k = e4m3_to_bf16(kr[h]); v = e4m3_to_bf16(vr[h]); }
      else { k = kr[h]; v = vr[h]; }
      if constexpr (decltype(careful)::value) v = finite_part<false>(v);
      const int key = key0 + 16 * h + srow;               // (keys before the window are in no row: their values are cleared)
      if (key < any_lo && key >= a.n_sink) v = u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4*>(&lds[buf][0][4096 * h + k_to]) = k;
      *reinterpret_cast<u32x4*>(&lds[buf][1][4096 * h + v_to]) = v;
    }
  };

  f32x16 o[4];
  float m, l;
  auto reset = [&]() {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
  };
  // one tile from a buffer; s: its weights
  auto attend = [&](int buf, int key0, const TilePages<KT>& pages, f32x16 (&s)[2]) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const u32x4 k = *reinterpret_cast<const u32x4*>(&lds[buf][0][8192 * kt + k_at + (k_swap ^ 32 * e)]);
        s[kt] = mfma32(k, q[e], s[kt]);
      }
    }
    bool good = true;
#pragma unroll
    for (int h = 0; h < KT / 16; ++h) good = good && page_ok(pages.id[h]);
    if (!(good && key0 + KT - 1 <= min_hi && (key0 >= max_lo || key0 + KT <= a.n_sink))) {
      // keys outside the row's set: key 32 kt + 8 (i / 4) + i % 4 of the tile, from this lane's first one on
      const int at = key0 + 4 * u, to = hi - at, from = lo - at, sink = a.n_sink - at;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 32 * kt + 8 * (i >> 2) + (i & 3);
          const bool ok = page_ok(pages.id[2 * kt + (i >> 3)]);
          s[kt][i] = ok && key <= to && (key >= from || key < sink) ? s[kt][i] : -INFINITY;
        }
    }
    float top = s[0][0];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kt][i]);
    top *= to_log2;
    if (__any(top > m + 8.f)) {
      const float m1 = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
      const float by = m == m1 ? 1.f : __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= by;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= by;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    u32x4 p[4];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[kt][i] = __builtin_amdgcn_exp2f(fmaf(s[kt][i], to_log2, -ref));
        l += s[kt][i];
        if (i & 1) p[2 * kt + (i >> 3)][(i & 7) >> 1] = pack_bf16(s[kt][i - 1], s[kt][i]);
      }
#pragma unroll
    for (int x = 0; x < 4; ++x)                            // sixteen keys
#pragma unroll
      for (int d = 0; d < 4; ++d) {                        // 32 elements
        const char* from = &lds[buf][1][4096 * x + v_at + ((d ^ quad) << 6)];
        const u32x2 v0 = read_transposed(from), v1 = read_transposed(from + 2048);
        o[d] = mfma32(u32x4{v0.x, v0.y, v1.x, v1.y}, p[x], o[d]);
      }
  };

  reset();
  if (t_begin < t_end) {
    TilePages<KT> now, next;
    tile_pages(t_begin, now);
    fetch(t_begin, now);
    if (t_begin + 1 < t_end) tile_pages(t_begin + 1, next);
    put(0, tile_key(t_begin), std::false_type{});
    __syncthreads();
#pragma unroll 1
    for (int v = t_begin; v < t_end; ++v) {
      const int buf = (v - t_begin) & 1, key0 = tile_key(v);
      TilePages<KT> after = next;
      if (v + 1 < t_end) fetch(v + 1, next);
      if (v + 2 < t_end) tile_pages(v + 2, after);
      if (key0 <= wave_hi) {
        f32x16 s[2];
        attend(buf, key0, now, s);
      }
      if (v + 1 < t_end) put(buf ^ 1, tile_key(v + 1), std::false_type{});
      __syncthreads();
      now = next;
      next = after;
    }
  }
  // An infinity or a NaN of V reaches rows that do not attend its key (a weight of 0 does not clear it) and leaves a NaN
  // there: a workgroup that ends with one goes over its tiles again, one at a time.  What is not finite is left out of the
  // products and added key by key to the rows that attend the key; weights change lanes through the other buffer.
  float sum = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += o[d][i];
  if (__syncthreads_or(sum != sum)) {
    reset();
    float* weights = reinterpret_cast<float*>(&lds[1][0][0]) + (32 * wave + c) * KT;
#pragma unroll 1
    for (int v = t_begin; v < t_end; ++v) {
      const int key0 = tile_key(v);
      TilePages<KT> now;
      tile_pages(v, now);
      fetch(v, now);
      put(0, key0, std::true_type{});
      __syncthreads();
      if (key0 <= wave_hi) {
        f32x16 s[2];
        attend(0, key0, now, s);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int i = 0; i < 16; ++i) weights[32 * kt + 8 * (i >> 2) + 4 * u + (i & 3)] = s[kt][i];
#pragma unroll 1
        for (int k = 0; k < KT; ++k) {
          const int key = key0 + k, id = table[min(key >> a.page_shift, a.max_pages - 1)];
          if (!page_ok(id) || key >= end) continue;
          const char* from = vbase + id * (a.v_page * kElem) + (uint32_t)(key & page_mask) * v_key;
          const bool attends = key <= hi && (key >= lo || key < a.n_sink);
          const float w = weights[k];
#pragma unroll
          for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int e = 32 * d + 8 * (i >> 2) + 4 * u + (i & 3);
              float y;
              if constexpr (ET == kFP8) y = fp8_to_float(reinterpret_cast<const uint8_t*>(from)[e]);
              else y = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(from)[e] << 16);
              if (attends && !(fabsf(y) < INFINITY)) o[d][i] += w * y;
            }
        }
      }
      __syncthreads();
    }
  }

  if (!real) return;
  l += __shfl_xor(l, 32);
  if (pc.pieces > 1) {
    const int64_t slot = pc.slot + pc.piece;
    if (slot >= a.slots) return;
    float* pp = a.partial + (slot * R + row) * kPartialRow;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(pp + 32 * d + 8 * i + 4 * u) = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    if (u == 0) { pp[128] = m; pp[129] = l; }
  } else {
    const int64_t to = (int64_t)(pc.r.row + first + t) * a.Hq + pc.g * a.G + head;
    const float by = l == 0.f ? 0.f : (a.v_scale ? a.v_scale[pc.g] : 1.f) / l;
    uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + to * kHeadDim + 4 * u;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x2*>(out + 32 * d + 8 * i) = u32x2{pack_bf16(o[d][4 * i] * by, o[d][4 * i + 1] * by),
                                                               pack_bf16(o[d][4 * i + 2] * by, o[d][4 * i + 3] * by)};
    if (a.lse && u == 0) a.lse[to] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
  }
}

}  // namespace

void launch_paged_many_rows(const PagedArgs& a, bool fp8, const PagedForm& form, hipStream_t s) {
  if (fp8) paged_many_rows_kernel<kFP8><<<(unsigned)form.pieces, 256, 0, s>>>(a);
  else paged_many_rows_kernel<kBF16><<<(unsigned)form.pieces, 256, 0, s>>>(a);
}

}  // namespace mp
