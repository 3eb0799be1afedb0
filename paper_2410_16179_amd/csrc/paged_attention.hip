// Exact attention over a paged key-value cache: the form for few rows per KV head, and the joining of pieces.
#include "paged_device.h"

#include <type_traits>

namespace mp {
namespace {

constexpr int kFewThreads = 64 * kPagedGroup;

// Joins the partials of a cut item, by one workgroup: groups of sixteen threads take a row of a KV head each, eight elements a thread, and
// where there are few rows several groups share a row's partials; eight partials are requested at once.  rows: of a head; all: of the set.  lds: room
// for as many rows as there are groups.
template <bool F32, int R, bool SETS, class Scale, class Finish>
__device__ inline void join_parts(const PagedArgs& a, float* lds, int first_share, int parts, int g0, int rows, int all, Scale scale_of, Finish finish) {
  constexpr int kAtOnce = 8, kLots = kFewThreads / 16;
  const int lot = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * 8;
  const int per_row = all < kLots ? kLots / all : 1;
  for (int base = 0; base == 0 || (SETS && base < all); base += kLots) {
    const int part = lot / all, n = base + lot - part * all, head = SETS && rows < all ? n / rows : 0, row = n - head * rows;   // (part 0 where a group has a row of its own)
    const bool busy = part < per_row && n < all;
    const float v_scale = busy ? scale_of(head) : 1.f;
    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    if (busy) {
      for (int p = part; p < parts; p += kAtOnce * per_row) {
        f32x2 x[kAtOnce][4], ml[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const int q = p + i * per_row;
          ml[i] = f32x2{-INFINITY, 0.f};
          if (q < parts) {
            const float* from = a.partial + ((2 * ((int64_t)(first_share + q) * a.Hkv + g0 + head) + (q == 0 ? 1 : 0)) * R + row) * kPartialRow;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = load_through(from + e0 + 2 * e);
            ml[i] = load_through(from + 128);
          }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, ml[i].x);
        if (top > -INFINITY) {
          const float by = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
          l *= by;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] *= by;
          m = top;
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            if (ml[i].x == -INFINITY) continue;            // (an empty partial, or none)
            const float b1 = ml[i].x == top ? 1.f : __builtin_amdgcn_exp2f(ml[i].x - top);
            l += b1 * ml[i].y;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += b1 * x[i][e >> 1][e & 1];
          }
        }
      }
    }
    if (per_row > 1) {
      float* to = lds + lot * kPartialRow;
      if (busy) {
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e0 + e] = o[e];
        if (e0 == 0) { to[128] = m; to[129] = l; }
      }
      __syncthreads();
      if (busy && part == 0) {
        for (int i = 1; i < per_row; ++i) {
          const float* from = lds + (lot + i * all) * kPartialRow;
          const float m1 = from[128], top = fmaxf(m, m1);
          if (m1 == -INFINITY) continue;
          const float b0 = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), b1 = m1 == top ? 1.f : __builtin_amdgcn_exp2f(m1 - top);
          l = b0 * l + b1 * from[129];
          m = top;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = b0 * o[e] + b1 * from[e0 + e];
        }
      }
    }
    if (busy && part == 0) finish(head, row, e0, o, m, l, v_scale);
  }
}

// Behind the wavefronts' parts in `joined`: the rows of the item they belong to are written, or, where other workgroups have keys of it
// too, a partial; the last of these workgroups joins the partials.
template <bool F32, int NR, bool SETS>
__device__ inline void finish_item(const PagedArgs& a, const PagedShare& share, const PagedItem& item,
                                   float (&joined)[kPagedGroup][16 * NR][kPartialRow], int& last_one) {
  constexpr int R = 16 * NR;
  const int tt = item.tile / a.head_blocks, hb = item.tile - tt * a.head_blocks;
  const int first = tt * a.tile_tokens, last = min(first + a.tile_tokens, item.r.tokens) - 1;
  const int rows = a.head_blocks > 1 ? min(a.G - hb * R, R) : (last - first + 1) * a.G;
  const int all = rows << item.shift, g0 = item.set << item.shift, waves = kPagedGroup >> item.shift;   // rows of the set; wavefronts of a KV head
  auto scale_of = [&](int head) { return a.v_scale ? a.v_scale[g0 + head] : 1.f; };
  auto finish = [&](int head, int row, int e0, const float (&o)[8], float m, float l, float v_scale) {
    const int t = a.head_blocks > 1 ? 0 : row / a.G, h = a.head_blocks > 1 ? hb * R + row : row - t * a.G, g = g0 + head;
    paged_write_row<F32>(a, (int64_t)(item.r.row + first + t) * a.Hq + g * a.G + h, e0, o, m, l, v_scale);
  };
  const bool whole = item.from == 0 && item.to == item.groups;
  const int e0 = (threadIdx.x & 15) * 8;
  for (int n = threadIdx.x >> 4; n < all; n += kFewThreads / 16) {
    const int head = SETS && item.shift ? n / rows : 0, row = n - head * rows;
    const float v_scale = scale_of(head);
    const float(*const part)[16 * NR][kPartialRow] = joined + head * waves;
    float m = -INFINITY;                                   // (of fewer than eight wavefronts some are looked at again: the same maximum)
#pragma unroll
    for (int w = 0; w < kPagedGroup; ++w) m = fmaxf(m, part[w & (waves - 1)][row][128]);
    float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, l = 0.f;
#pragma unroll
    for (int w = 0; w < kPagedGroup; ++w) {
      if (SETS && w >= waves) break;                       // (not taken again with a weight of 0: an output may be infinite)
      const float mw = part[w][row][128];
      const float by = mw == -INFINITY ? 0.f : (mw == m ? 1.f : __builtin_amdgcn_exp2f(mw - m));
      l += by * part[w][row][129];
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] += by * part[w][row][e0 + e];
    }
    if (whole) {
      finish(head, row, e0, o, m, l, v_scale);
    } else {
      const int slot = 2 * (share.j * a.Hkv + g0 + head) + (item.from == 0 ? 1 : 0);
      float* pp = a.partial + ((int64_t)slot * R + row) * kPartialRow;
#pragma unroll
      for (int e = 0; e < 8; e += 2) store_through(pp + e0 + e, o[e], o[e + 1]);
      if (e0 == 0) store_through(pp + 128, paged_partial_max(m, l), l);
    }
  }
  if (whole) return;
  const int first_share = item.from == 0 ? share.j : item.begin / share.each;
  const int parts = (item.begin + item.groups - 1) / share.each - first_share + 1;
  unsigned* const arrived = a.arrived + first_share * (a.Hkv >> item.shift) + item.set;
  stored();
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned before = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last_one = before + 1 == (unsigned)parts;
    if (last_one) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last_one) return;
  join_parts<F32, R, SETS>(a, &joined[0][0][0], first_share, parts, g0, rows, all, scale_of, finish);
}

// ---- few rows ------------------------------------------------------------------------------------
// A wavefront attends tiles of KT keys with up to 16 NR query rows.  Scores are formed transposed,
// S^T = K Q^T: MFMA A = 16 keys (lane c = lane % 16 holds a key, the lane's quarter u = lane / 16 a quarter of its
// elements; loaded by quads of lanes, 64 bytes of a key at a time, which then change lanes), B = the query rows, so a lane ends up with four keys of one row
// per MFMA: the row's maximum, its weights and its output live in the lanes of one column c.  The output
// is transposed too, O^T = V^T P^T: B = the weights exactly where the first product left them (the order of
// the summed keys is free as long as A has the same), A = V with lane c holding elements 8c .. 8c + 7 of
// eight keys: sixteen lanes read a whole row, and one v_perm per register pairs two keys' elements.
// Neither K nor V passes through LDS.
// bf16 weights are taken as a sum of two bf16 (2^-17): the matrix unit has time, the output is rounded once.
// Bound by memory.  One workgroup per compute unit, equal shares of the keys: 16 requests of 65536 keys (bf16, 4.3 GB) take 634 us, 6.77 TB/s,
// the rate of a plain read; 48 ragged ones in e4m3 (491 MB) 102, 4.8 TB/s; 6 in float32 (652 MB) 113, 5.8 TB/s.  One of 98304 keys (403 MB) 75: 60
// at that rate, the rest is what one of 2048 keys takes, 12 us: launch, the way to the first keys, the join (2 to 4 us).
// Four bits: a wavefront takes 64 keys at once (128: 48 ragged requests of up to 30011 keys 97 | 106 us, 2048 keys 14.2 | 17.1).  16 requests of 65536 keys (1.14 GB)
// take 191 to 202 us, 5.6 to 6.0 TB/s (24 without a pause 193 to 242): widening keys and values to bf16 and pairing them are 128 and 64 of 400 vector instructions for 64 keys, and two wavefronts a SIMD
// issue one in four cycles each; with a descriptor multiplied out for every 16 keys, 350 scalar ones more, 212.
// Shares in the same launch against pieces and a second kernel (four wavefronts a workgroup): 2048 keys 14.6 -> 12.8 us, e4m3 ragged 186 -> 107.
// 384, 512 or 768 smaller workgroups were slower.
//
// m: running maximum (log2 units) of the column's row, raised only when a tile exceeds it by 8
// (weights stay below 2^8; the sum and the output are float32), so most tiles need no rescaling and no
// exchange between lanes.  l: this lane's share of the sum.
template <int ET, int NR>
struct FewRows {
  static constexpr bool kF32 = ET == kFP32;
  static constexpr int kTile = kF32 ? 16 : (ET == kFP4 ? kPagedFourTile : 32);   // keys per tile
  static constexpr int kHalves = kTile / 16;
  static constexpr int kFrags = ET == kFP4 ? 4 : 8;      // loads of a lane per tile for V, and for K, which e4m3 takes 16 elements at a time
  static constexpr int kKeyFrags = ET == kFP8 || ET == kFP4 ? 4 : 8;
  typedef typename std::conditional<ET == kFP8, u32x2, u32x4>::type Raw;

  u32x4 q[NR][kF32 ? 8 : 4];                             // query rows, as the B operand
  f32x4 o[NR][8];
  float m[NR], l[NR];
  u32x4 kf[kKeyFrags];
  Raw vf[kFrags];
  uint32_t ks[ET == kFP4 ? kHalves : 1], vs[ET == kFP4 ? kHalves : 1];   // four bits: scales as they come
};

template <int ET, int NR, bool SETS>
__global__ __launch_bounds__(kFewThreads, 2) void paged_few_rows_kernel(const PagedArgs a) {
  using F = FewRows<ET, NR>;
  constexpr bool kF32 = F::kF32, kFour = ET == kFP4;
  constexpr int KT = F::kTile, R = 16 * NR;
  constexpr int kElem = ET == kFP32 ? 4 : (ET == kFP8 ? 1 : 2);   // (not of kFP4)
  __shared__ float joined[kPagedGroup][R][kPartialRow];
  __shared__ int last_one;

  // Where the workgroup is in its share lies in LDS: kept in registers over the loops below it would cost them their own.
  __shared__ PagedShare at_share;
  {
    PagedShare share;
    if (!paged_share<KT, SETS>(a, blockIdx.x, share)) return;
    if (threadIdx.x == 0) at_share = share;
  }
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll 1
  for (;;) {
  // (unknown to the compiler, so that what follows from it is worked out per item and not kept in registers over all of them)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, c = lane & 15, u = lane >> 4;
  const PagedItem item = paged_item<KT, SETS>(a, at_share);
  const PagedRequest req = item.r;
  // the wavefront's KV head, and its place among the wavefronts that share the head's tiles
  const int waves = kPagedGroup >> item.shift, place = wave & (waves - 1);
  const int tile = item.tile, g = (item.set << item.shift) + (wave >> (kPagedGroupShift - item.shift));
  const int len = req.len, tokens = req.tokens;
  const int tt = tile / a.head_blocks, hb = tile - tt * a.head_blocks;
  const int first = tt * a.tile_tokens, last = min(first + a.tile_tokens, tokens) - 1;
  const int heads = min(a.G - hb * R, R);                // query heads of the tile: all G where a tile holds whole tokens
  const int rows = a.head_blocks > 1 ? heads : (last - first + 1) * a.G;
  const PagedSpan span = paged_span<KT>(a, len, tokens, first, last);
  const int t_begin = item.from << item.group_shift, t_end = min(item.to << item.group_shift, span.count);
  // row of this lane's column: token and head
  int hi[NR], lo[NR];                                    // keys it attends: [lo, hi], and those below n_sink
  F f{};                                                 // (all of it: what an earlier item left would stay in registers)
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    const int row = c + 16 * n;
    const int t = a.head_blocks > 1 ? 0 : row / a.G, h = a.head_blocks > 1 ? hb * R + row : row - t * a.G;
    const bool ok = row < rows;
    hi[n] = ok ? len - tokens + first + t : -1;
    lo[n] = a.n_local > 0 ? hi[n] - a.n_local + 1 : 0;
    const int64_t at = (int64_t)(req.row + first + t) * a.q_t + (int64_t)(g * a.G + h) * a.q_h;
#pragma unroll
    for (int s = 0; s < (kF32 ? 8 : 4); ++s) {
      f.q[n][s] = u32x4{0, 0, 0, 0};
      if (ok) {
        const int e = kF32 ? 64 * (s >> 2) + 16 * u + 4 * (s & 3) : 32 * u + 8 * s;
        if (kF32) f.q[n][s] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(a.q) + at + e);
        else f.q[n][s] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + at + e);
      }
    }
  }
  const int min_hi = len - tokens + first;               // what every row of the tile attends: [max_lo, min_hi]
  const int max_lo = a.n_local > 0 ? len - tokens + last - a.n_local + 1 : 0;
  const int end = len - tokens + last + 1;               // behind what some row attends
  const float to_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[g] : 1.f);

  const const_i32_ptr table = (const_i32_ptr)(a.table + (int64_t)item.b * a.max_pages);
  const char* kbase = reinterpret_cast<const char*>(a.k) + pool_bytes<ET>((int64_t)g * a.k_head);
  const char* vbase = reinterpret_cast<const char*>(a.v) + pool_bytes<ET>((int64_t)g * a.v_head);
  const int page_mask = (1 << a.page_shift) - 1;
  const uint32_t k_key = (uint32_t)pool_bytes<ET>(a.k_key), v_key = (uint32_t)pool_bytes<ET>(a.v_key);
  // This lane's place in 16 keys.  K: a quad of lanes takes keys 4 (c / 4) + i, one (e4m3: two) at a time, of which each lane
  // 16 bytes; V: keys 4u .. 4u + 3.
  const int quad = c >> 2, in_quad = c & 3;
  const bool odd = c & 1, upper = c & 2;
  uint32_t k_lane = (ET == kFP8 ? 4 * quad + (in_quad >> 1) : 4 * quad) * k_key +
                    (ET == kFP8 ? 32 * u + 16 * (in_quad & 1) : 64 * u + 16 * in_quad);
  uint32_t v_lane = 4 * u * v_key + (kF32 ? 16 * c : 8 * c * kElem);
  // Four bits: sixteen rows of 64 bytes are one load, a quad of lanes to a row; rows change lanes through the wavefront's own part of LDS (K in its
  // first 4096 bytes, V in the next, V's scales behind them), where lane 4 r + p leaves what it has at 16 times its number: chunk p ^ (r / 4) of
  // row r, so that lanes which read a chunk of 16 rows, or one of rows 4u + j, meet different banks.
  char* const exchange = reinterpret_cast<char*>(&joined[wave][0][0]);
  if constexpr (kFour) {
    k_lane = (lane >> 2) * k_key + 16 * (in_quad ^ u);
    v_lane = (lane >> 2) * v_key + 16 * (in_quad ^ u);
  }
  const char* const ksbase = reinterpret_cast<const char*>(a.k_block) + ((int64_t)g * a.k_head >> 5);
  const char* const vsbase = reinterpret_cast<const char*>(a.v_block) + ((int64_t)g * a.v_head >> 5);
  const uint32_t ks_key = (uint32_t)(a.k_key >> 5), vs_key = (uint32_t)(a.v_key >> 5);
  const bool one_page = kFour && (KT >> a.page_shift) <= 1;   // whether a tile lies in one
  // Four bits, where addresses weigh more than elsewhere: in rows of 128 elements (64 bytes of a pool, four of its scales) from the head's first one on.
  auto row_of = [&](int id, int at, uint32_t page_rows, uint32_t key_rows) {
    return (uint64_t)(uint32_t)id * page_rows + (uint32_t)at * key_rows;
  };
  uint64_t k_row[kFour ? F::kHalves : 1];                // of the tile that is requested; V's where the pools have the same strides

  auto tile_key = [&](int v) { return (v < span.sink ? v : v + span.skip) * KT; };
  auto tile_pages = [&](int v, TilePages<KT>& p) {
    const int key0 = tile_key(v);
    if (one_page) {
      const int at = key0 >> a.page_shift, id = table[at < a.max_pages ? at : a.max_pages - 1];
#pragma unroll
      for (int h = 0; h < F::kHalves; ++h) p.id[h] = id;
      return;
    }
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) {
      const int at = (key0 + 16 * h) >> a.page_shift;
      p.id[h] = table[at < a.max_pages ? at : a.max_pages - 1];
    }
  };
  auto page_ok = [&](int id) { return (uint32_t)id < (uint32_t)a.n_pages; };
  auto descriptor = [&](const char* base, uint64_t offset, int rows, uint32_t stride) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + offset), 0, rows * stride, kBufferWord3);
  };
  // (four bits: where a workgroup takes neighbouring heads their rows share lines)
  auto load_four = [&](__amdgpu_buffer_rsrc_t rows, uint32_t at, u32x4& to) {
    if constexpr (SETS) load_shared(rows, at, to);
    else load_once(rows, at, to);
  };
  auto request_k = [&](int key0, const TilePages<KT>& p, const int (&valid)[F::kHalves]) {
    if constexpr (kFour) {
      if (one_page) {
        int there = 0;
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h) there += valid[h];
        const uint64_t row = row_of(there ? p.id[0] : 0, key0 & page_mask, a.k_page_rows, a.k_key_rows);
        const auto rows = descriptor(kbase, row * 64, there, k_key), scales = descriptor(ksbase, row * 4, there, ks_key);
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h) {
          load_four(rows, k_lane + 16 * h * k_key, f.kf[h]);
          f.ks[h] = load_byte(scales, (16 * h + c) * ks_key + u);
        }
        k_row[0] = row;
        return;
      }
    }
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) {
      if constexpr (kFour) {
        k_row[h] = row_of(valid[h] ? p.id[h] : 0, (key0 + 16 * h) & page_mask, a.k_page_rows, a.k_key_rows);
        load_four(descriptor(kbase, k_row[h] * 64, valid[h], k_key), k_lane, f.kf[h]);
        f.ks[h] = load_byte(descriptor(ksbase, k_row[h] * 4, valid[h], ks_key), c * ks_key + u);
      } else {
      const auto rows = rows16(kbase, pool_bytes<ET>(a.k_page), k_key, p.id[h], (key0 + 16 * h) & page_mask, valid[h]);
#pragma unroll
      for (int i = 0; i < F::kKeyFrags / F::kHalves; ++i) {
        const uint32_t at = ET == kFP8 ? 2 * i * k_key : (i & 3) * k_key + 256 * (i >> 2);
        load_once(rows, k_lane + at, f.kf[h * (F::kKeyFrags / F::kHalves) + i]);
      }
      }
    }
  };
  // (behind request_k of the same tile)
  auto request_v = [&](int key0, const TilePages<KT>& p, const int (&valid)[F::kHalves]) {
    if constexpr (kFour) {
      if (one_page) {
        int there = 0;
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h) there += valid[h];
        const uint64_t row = a.same_strides ? k_row[0] : row_of(there ? p.id[0] : 0, key0 & page_mask, a.v_page_rows, a.v_key_rows);
        const auto rows = descriptor(vbase, row * 64, there, v_key), scales = descriptor(vsbase, row * 4, there, vs_key);
#pragma unroll
        for (int h = 0; h < F::kHalves; ++h) {
          load_four(rows, v_lane + 16 * h * v_key, f.vf[h]);
          load_shared(scales, (16 * h + c) * vs_key, f.vs[h]);
        }
        return;
      }
    }
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) {
      if constexpr (kFour) {
        const uint64_t row = a.same_strides ? k_row[h] : row_of(valid[h] ? p.id[h] : 0, (key0 + 16 * h) & page_mask, a.v_page_rows, a.v_key_rows);
        load_four(descriptor(vbase, row * 64, valid[h], v_key), v_lane, f.vf[h]);
        load_shared(descriptor(vsbase, row * 4, valid[h], vs_key), c * vs_key, f.vs[h]);
      } else {
      const auto rows = rows16(vbase, pool_bytes<ET>(a.v_page), v_key, p.id[h], (key0 + 16 * h) & page_mask, valid[h]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (kF32) {
#pragma unroll
          for (int d = 0; d < 2; ++d) load_once(rows, v_lane + j * v_key + 256 * d, f.vf[2 * j + d]);
        } else {
          load_once(rows, v_lane + j * v_key, f.vf[4 * h + j]);
        }
      }
      }
    }
  };
  constexpr int kScores = 4 * F::kHalves;                // of a lane: key 16 (i / 4) + 4 u + i % 4 of the tile is number i
  auto scores = [&](float (&s)[NR][kScores]) {
    // a key per lane: its elements 32 u .. 32 u + 31 (float32: 16 u .. 16 u + 15 of both halves of the row)
    if constexpr (kFour) {
#pragma unroll
      for (int h = 0; h < F::kHalves; ++h) *reinterpret_cast<u32x4*>(exchange + 1024 * h + 16 * lane) = f.kf[h];
      in_order();
#pragma unroll
      for (int h = 0; h < F::kHalves; ++h) f.kf[h] = *reinterpret_cast<const u32x4*>(exchange + 1024 * h + 64 * c + 16 * (u ^ quad));
      in_order();
    } else if constexpr (ET == kFP8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) join_halves(f.kf[2 * h], f.kf[2 * h + 1], upper);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) transpose_quads(f.kf[4 * h], f.kf[4 * h + 1], f.kf[4 * h + 2], f.kf[4 * h + 3], odd, upper);
    }
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) {
      f32x4 acc[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int n = 0; n < NR; ++n)
              acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(f.kf[i][e]), __uint_as_float(f.q[n][i][e]), acc[n], 0, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4 k;
          if constexpr (kFour) {
            k = e2m1_to_bf16(f.kf[h][i], f.ks[h] << 23);
          } else if constexpr (ET == kFP8) {
            const u32x4 w = f.kf[2 * h + (i >> 1)];
            k = e4m3_to_bf16(i & 1 ? u32x2{w.z, w.w} : u32x2{w.x, w.y});
          } else {
            k = f.kf[4 * h + i];
          }
#pragma unroll
          for (int n = 0; n < NR; ++n) acc[n] = mfma_bf16(k, f.q[n][i], acc[n]);
        }
      }
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][4 * h + i] = acc[n][i] * to_log2;
    }
  };
  // scores -> weights, in place; the state is raised where they ask for it
  auto weigh = [&](float (&s)[NR][kScores]) {
    bool raise = false;
    float top[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      top[n] = s[n][0];
#pragma unroll
      for (int i = 1; i < kScores; ++i) top[n] = fmaxf(top[n], s[n][i]);
      raise = raise || top[n] > f.m[n] + 8.f;
    }
    if (__any(raise)) {
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float t = fmaxf(top[n], __shfl_xor(top[n], 16));
        t = fmaxf(t, __shfl_xor(t, 32));
        const float m1 = fmaxf(f.m[n], t);
        const float by = f.m[n] == m1 ? 1.f : __builtin_amdgcn_exp2f(f.m[n] - m1);
        f.m[n] = m1;
        f.l[n] *= by;
#pragma unroll
        for (int t8 = 0; t8 < 8; ++t8) f.o[n][t8] *= by;
      }
    }
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const float ref = f.m[n] == -INFINITY ? 0.f : f.m[n];
#pragma unroll
      for (int i = 0; i < kScores; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(s[n][i] - ref);
        f.l[n] += s[n][i];
      }
    }
  };
  // (of the weights those from `at` on)
  auto add_values = [&](const float (&s)[NR][kScores], const u32x4 (&v)[8], int at0) {
    if constexpr (kF32) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              f.o[n][4 * d + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[2 * i + d][e]), s[n][i], f.o[n][4 * d + e], 0, 0, 0);
    } else {
      u32x4 ph[NR], pl[NR];                              // a weight as two bf16
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s0 = s[n][at0 + 2 * i], s1 = s[n][at0 + 2 * i + 1];
          ph[n][i] = pack_bf16(s0, s1);
          pl[n][i] = pack_bf16(s0 - __uint_as_float(ph[n][i] << 16), s1 - __uint_as_float(ph[n][i] & 0xffff0000u));
        }
#pragma unroll
      for (int t8 = 0; t8 < 8; ++t8) {                   // V^T of elements 8 c + t8, two keys a register
        const uint32_t pick = t8 & 1 ? 0x07060302u : 0x05040100u;
        u32x4 at;
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = __builtin_amdgcn_perm(v[2 * i + 1][t8 >> 1], v[2 * i][t8 >> 1], pick);
#pragma unroll
        for (int n = 0; n < NR; ++n) f.o[n][t8] = mfma_bf16(at, pl[n], mfma_bf16(at, ph[n], f.o[n][t8]));
      }
    }
  };
  // Four bits: V into LDS, from where values() takes 32 keys at a time, those from 32 `group` on.
  auto stage_v = [&]() {
    if constexpr (kFour) {
#pragma unroll
      for (int h = 0; h < F::kHalves; ++h) *reinterpret_cast<u32x4*>(exchange + 4096 + 1024 * h + 16 * lane) = f.vf[h];
      const uint32_t lower = u & 1 ? f.vs[1] : f.vs[0], higher = u & 1 ? f.vs[3] : f.vs[2];
      *reinterpret_cast<uint32_t*>(exchange + 8192 + 4 * lane) = u & 2 ? higher : lower;
      in_order();
    }
  };
  auto values = [&](u32x4 (&v)[8], int group) {
    if constexpr (kFour) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4 scale = *reinterpret_cast<const u32x4*>(exchange + 8192 + 64 * (2 * group + h) + 16 * u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(exchange + 4096 + 1024 * (2 * group + h) + 64 * (4 * u + j) + 16 * (quad ^ u) + 4 * in_quad);
          v[4 * h + j] = e2m1_to_bf16(w, rotate_right(scale[j], to_scale(quad)));
        }
      }
      return;
    } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (ET == kFP8) v[i] = e4m3_to_bf16(f.vf[i]);
      else v[i] = f.vf[i];
    }
    }
  };
  constexpr int kGroups = kFour ? 2 : 1;                 // of keys, in which the values are taken

  // whether every row attends all keys of a tile
  auto in_full = [&](int v) {
    const int key0 = tile_key(v);
    return key0 + KT - 1 <= min_hi && (key0 >= max_lo || key0 + KT <= a.n_sink);
  };
  auto pages_ok = [&](const TilePages<KT>& p) {
    bool ok = true;
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) ok = ok && page_ok(p.id[h]);
    return ok;
  };
  bool bad_page = false;
  // the first such tile from v on with pages that are there; they are read
  auto find = [&](int v, TilePages<KT>& p) {
    for (; v < t_end; v += waves) {
      if (!in_full(v)) continue;
      tile_pages(v, p);
      if (pages_ok(p)) break;
      bad_page = true;
    }
    return v;
  };
  // rows of the tile's halves that are there
  auto valid_rows = [&](int key0, const TilePages<KT>& p, int (&valid)[F::kHalves]) {
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) valid[h] = page_ok(p.id[h]) ? min(max(end - key0 - 16 * h, 0), 16) : 0;
  };
  // keys outside the rows' sets get no weight
  auto mask = [&](int key0, const int (&valid)[F::kHalves], float (&s)[NR][kScores]) {
#pragma unroll
    for (int h = 0; h < F::kHalves; ++h) {
      const int at = key0 + 16 * h + 4 * u;               // key i of this lane is at + i
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        const int to = valid[h] ? hi[n] - at : -1, from = lo[n] - at, sink = a.n_sink - at;
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][4 * h + i] = i <= to && (i >= from || i < sink) ? s[n][4 * h + i] : -INFINITY;
      }
    }
  };
  TilePages<KT> now{}, next{}, after{};
  auto reset = [&]() {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int t8 = 0; t8 < 8; ++t8) f.o[n][t8] = f32x4{0.f, 0.f, 0.f, 0.f};
      f.m[n] = -INFINITY;
      f.l[n] = 0.f;
    }
  };
  reset();
  // The tiles, whole ones and then the others (the last ones, the borders of the window and of the sink): the next one's K is requested
  // when the scores have taken this one's, its V behind the products with this one's.
  auto other = [&](int v) {                               // the first of the others from v on
    while (v < t_end && in_full(v)) v += waves;
    return v;
  };
  int w = t_begin + place;
  if (a.n_local == 0) {                                   // (only from the first key on that some row does not attend)
    const int from = (min_hi + 1 > 0 ? min_hi + 1 : 0) / KT;
    if (from > w) w += (from - w + waves - 1) & ~(waves - 1);
  }
  w = other(w);
  TilePages<KT> w_pages{};
  if (w < t_end) tile_pages(w, w_pages);
  int v = find(t_begin + place, now), v1 = t_end;
  int valid[F::kHalves];
  {
    const int first_tile = v < t_end ? v : w;
    if (first_tile < t_end) {
      const int key0 = tile_key(first_tile);
      const TilePages<KT> p = v < t_end ? now : w_pages;
      valid_rows(key0, p, valid);
      request_k(key0, p, valid);
      request_v(key0, p, valid);
    }
  }
  if (v < t_end) v1 = find(v + waves, next);
#pragma unroll 1
  while (v < t_end) {
    const int v2 = v1 + waves, ahead = v1 < t_end ? v1 : w;
    if (v2 < t_end) tile_pages(v2, after);
    const int key1 = tile_key(ahead);
    const TilePages<KT> p = v1 < t_end ? next : w_pages;
    float s[NR][kScores];
    scores(s);
    if (ahead < t_end) {
      valid_rows(key1, p, valid);
      request_k(key1, p, valid);
    }
    if constexpr (kFour) {
      stage_v();
      if (ahead < t_end) request_v(key1, p, valid);
    }
    weigh(s);
#pragma unroll
    for (int x = 0; x < kGroups; ++x) {
      u32x4 vb[8];
      values(vb, x);
      add_values(s, vb, 8 * x);
    }
    if constexpr (!kFour) {
      if (ahead < t_end) request_v(key1, p, valid);
    }
    v = v1;
    v1 = v2;
    next = after;
    if (v1 < t_end && !(in_full(v1) && pages_ok(next))) {
      bad_page = bad_page || in_full(v1);
      v1 = find(v1 + waves, next);
    }
  }
#pragma unroll 1
  while (w < t_end) {
    const int key0 = tile_key(w), w1 = other(w + waves);
    TilePages<KT> p{};
    if (w1 < t_end) tile_pages(w1, p);
    float s[NR][kScores];
    scores(s);
    mask(key0, valid, s);
    if (w1 < t_end) {
      valid_rows(tile_key(w1), p, valid);
      request_k(tile_key(w1), p, valid);
    }
    if constexpr (kFour) {
      stage_v();
      if (w1 < t_end) request_v(tile_key(w1), p, valid);
    }
    weigh(s);
#pragma unroll
    for (int x = 0; x < kGroups; ++x) {
      u32x4 vb[8];
      values(vb, x);
      add_values(s, vb, 8 * x);
    }
    if constexpr (!kFour) {
      if (w1 < t_end) request_v(tile_key(w1), p, valid);
    }
    w = w1;
  }

  // The products take every row of a tile with every key's V: an infinity or a NaN there reaches rows that do not attend the key
  // (a weight of 0 does not clear it), and an infinity may come out as a NaN (the two parts of a weight differ in sign).
  // Either leaves a NaN in the output, so a wavefront that ends with one goes over its tiles again, carefully: what is
  // not finite is left out of the products and added afterwards to the rows that attend its key.  So does one that met a page that is none.
  float sum = 0.f;                                       // NaN if one of them is, or if infinities meet
#pragma unroll
  for (int n = 0; n < NR; ++n)
#pragma unroll
    for (int t8 = 0; t8 < 8; ++t8) sum += (f.o[n][t8][0] + f.o[n][t8][1]) + (f.o[n][t8][2] + f.o[n][t8][3]);
  if (bad_page || __any(sum != sum)) {
    reset();
#pragma unroll 1
    for (int v = t_begin + place; v < t_end; v += waves) {
      const int key0 = tile_key(v);
      tile_pages(v, now);
      valid_rows(key0, now, valid);
      request_k(key0, now, valid);
      request_v(key0, now, valid);
      float s[NR][kScores];
      scores(s);
      mask(key0, valid, s);
      stage_v();
      weigh(s);
      uint32_t cleared = 0;
#pragma unroll
      for (int group = 0; group < kGroups; ++group) {
        u32x4 vb[8];
        values(vb, group);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const u32x4 x = finite_part<kF32>(vb[i]), d = x ^ vb[i];
          cleared |= d.x | d.y | d.z | d.w;
          vb[i] = x;
        }
        add_values(s, vb, 8 * group);
      }
      if (!__any(cleared != 0)) continue;
      if constexpr (kFour) in_order();
      // (the weights change lanes through LDS)
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < kScores; ++i) joined[wave][c + 16 * n][16 * (i >> 2) + 4 * u + (i & 3)] = s[n][i];
#pragma unroll 1
      for (int k = 0; k < KT; ++k) {
        const int key = key0 + k;
        int id = F::kHalves == 2 && k >= 16 ? now.id[F::kHalves - 1] : now.id[0];
        if constexpr (F::kHalves == 4) id = k >= 32 ? (k >= 48 ? now.id[3] : now.id[2]) : (k >= 16 ? now.id[1] : now.id[0]);
        if (!page_ok(id) || key >= end) continue;
        const char* row = vbase + id * pool_bytes<ET>(a.v_page) + (uint32_t)(key & page_mask) * v_key;
#pragma unroll
        for (int i = 0; i < (kF32 ? 8 : 4); ++i) {          // four elements at a time, or eight
          float x[8];
          if constexpr (kF32) {
            const float4 w = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(row) + 64 * (i >> 2) + 16 * u + 4 * (i & 3));
            x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
          } else if constexpr (kFour) {
            const uint32_t scale = reinterpret_cast<const uint8_t*>(vsbase + id * (a.v_page >> 5) + (uint32_t)(key & page_mask) * vs_key)[u];
            const u32x4 w = e2m1_to_bf16(*reinterpret_cast<const uint32_t*>(row + 16 * u + 4 * i), scale << 23);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
          } else {
            load8<ET>(row, 32 * u + 8 * i, x);
          }
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const float w = joined[wave][c + 16 * n][k];
            const bool attends = key <= hi[n] && (key >= lo[n] || key < a.n_sink);
#pragma unroll
            for (int e = 0; e < (kF32 ? 4 : 8); ++e) {
              const int t8 = kF32 ? 4 * (i >> 2) + e : e;
              if (attends && !(fabsf(x[e]) < INFINITY)) f.o[n][t8][i & 3] += w * x[e];
            }
          }
        }
      }
    }
  }

  // the wavefronts' parts, joined in LDS
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float l = f.l[n];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    float* to = joined[wave][c + 16 * n];
    if (kF32) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(to + 64 * d + 16 * u + 4 * i) =
              f32x4{f.o[n][4 * d][i], f.o[n][4 * d + 1][i], f.o[n][4 * d + 2][i], f.o[n][4 * d + 3][i]};
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 0; d < 2; ++d)
          *reinterpret_cast<f32x4*>(to + 32 * u + 8 * i + 4 * d) =
              f32x4{f.o[n][4 * d][i], f.o[n][4 * d + 1][i], f.o[n][4 * d + 2][i], f.o[n][4 * d + 3][i]};
    }
    if (u == 0) { to[128] = f.m[n]; to[129] = l; }
  }
  const PagedItem done = paged_item<KT, SETS>(a, at_share);      // (read before the barrier: behind it the first thread goes on to the next item)
  __syncthreads();
  finish_item<kF32, NR, SETS>(a, at_share, done, joined, last_one);
  if (wave == 0) paged_next<KT, SETS>(a, at_share);
  __syncthreads();
  if (at_share.pos >= at_share.end) return;
  }
}

// ---- joining the pieces of an item (many rows) --------------------------------------------------------
// A workgroup takes half of the rows of a cut item, sixteen lanes a row, eight elements a lane, four partials requested at once.
// (A workgroup per row, most of them without work, took 35 us of four prompts; two per item take 4.8 where nothing is cut.)
constexpr int kJoinThreads = 16 * kPagedManyRows / 2;
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(const PagedArgs a) {
  constexpr int KT = kPagedManyKeys, R = kPagedManyRows;
  __shared__ PagedPiece cut;
  __shared__ bool found;
  if (threadIdx.x < 64) {                                  // (one wavefront looks for all sixteen)
    PagedPiece pc;
    const bool there = paged_locate<KT, kCutItems>(a, blockIdx.x, pc);
    if (threadIdx.x == 0) { cut = pc; found = there; }
  }
  __syncthreads();
  if (!found) return;
  const PagedPiece pc = cut;
  const int row = blockIdx.y * (R / 2) + (threadIdx.x >> 4), e0 = (threadIdx.x & 15) * 8;
  const int tt = pc.tile / a.head_blocks, hb = pc.tile - tt * a.head_blocks;
  const int first = tt * a.tile_tokens, last = min(first + a.tile_tokens, pc.r.tokens) - 1;
  const int rows = a.head_blocks > 1 ? min(a.G - hb * R, R) : (last - first + 1) * a.G;
  if (row >= rows || pc.slot + pc.pieces > a.slots) return;
  const float* pp = a.partial + ((int64_t)pc.slot * R + row) * kPartialRow;
  const int64_t step = (int64_t)R * kPartialRow;
  float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int p = 0; p < pc.pieces; p += 4) {
    f32x4 x[4], y[4];
    f32x2 ml[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ml[i] = f32x2{-INFINITY, 0.f};
      if (p + i < pc.pieces) {
        const float* from = pp + (p + i) * step;
        x[i] = *reinterpret_cast<const f32x4*>(from + e0);
        y[i] = *reinterpret_cast<const f32x4*>(from + e0 + 4);
        ml[i] = *reinterpret_cast<const f32x2*>(from + 128);
      }
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, ml[i].x);
    if (top == -INFINITY) continue;
    const float by = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
    l *= by;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] *= by;
    m = top;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (ml[i].x == -INFINITY) continue;                  // (an empty partial, or none)
      const float b1 = ml[i].x == top ? 1.f : __builtin_amdgcn_exp2f(ml[i].x - top);
      l += b1 * ml[i].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) { o[e] += b1 * x[i][e]; o[4 + e] += b1 * y[i][e]; }
    }
  }
  const int t = a.head_blocks > 1 ? 0 : row / a.G, h = a.head_blocks > 1 ? hb * R + row : row - t * a.G;
  paged_write_row<false>(a, (int64_t)(pc.r.row + first + t) * a.Hq + pc.g * a.G + h, e0, o, m, l, a.v_scale ? a.v_scale[pc.g] : 1.f);
}

template <int ET, int NR>
hipError_t launch_few_rows(const PagedArgs& a, const PagedForm& form, hipStream_t s) {
  if (form.set_shift > 0) paged_few_rows_kernel<ET, NR, true><<<(unsigned)form.pieces, kFewThreads, 0, s>>>(a);
  else paged_few_rows_kernel<ET, NR, false><<<(unsigned)form.pieces, kFewThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attention(const PagedArgs& a, int element, const PagedForm& form, hipStream_t s) {
  if (element == kFP32) return launch_few_rows<kFP32, 1>(a, form, s);
  if (form.rows == kPagedManyRows) {
    launch_paged_many_rows(a, element, form, s);
    if (form.units > 0) paged_join_kernel<<<dim3((unsigned)form.units, 2), kJoinThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  if (element == kFP4) return form.rows == 16 ? launch_few_rows<kFP4, 1>(a, form, s) : launch_few_rows<kFP4, 2>(a, form, s);
  if (form.rows == 16) return element == kFP8 ? launch_few_rows<kFP8, 1>(a, form, s) : launch_few_rows<kBF16, 1>(a, form, s);
  return element == kFP8 ? launch_few_rows<kFP8, 2>(a, form, s) : launch_few_rows<kBF16, 2>(a, form, s);
}

}  // namespace mp
