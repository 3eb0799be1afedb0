// Exact attention over a paged key-value cache: the form for many rows per KV head (prompts, chunks of prompts).
#include "paged_device.h"

#include <type_traits>

namespace mp {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

constexpr int KT = kPagedManyKeys, R = kPagedManyRows;
constexpr int kTileBytes = KT * kHeadDim * 2;             // a tile of keys or values as bf16
constexpr int kAhead = 2;                                // operands read ahead of their product

__device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Four values of this lane's column, from a block of four rows by sixteen columns that sixteen lanes point at.
__device__ inline u32x2 read_transposed(const char* lds) {
  typedef i16x4 __attribute__((address_space(3))) * lds_ptr;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds)));
}

// f(BEGIN), .. f(END - 1), as constants
template <int BEGIN, int END, class F>
__device__ inline void each(F&& f) {
  if constexpr (BEGIN < END) {
    f(std::integral_constant<int, BEGIN>{});
    each<BEGIN + 1, END>(f);
  }
}

// Four wavefronts share tiles of 64 keys in LDS (two buffers); each has 32 query rows.  As in the form for few rows
// both products are formed transposed, here with the 32 x 32 x 16 MFMA: S^T = K Q^T has keys along an
// accumulator's registers and a query row in a lane (and the lane 32 further on), so maximum, weights and sum need
// no exchange but one between two lanes, and the weights are the B operand of O^T = V^T P^T as they are.
// A operands come from LDS: K rows by 16-byte reads, V^T by the transposing read, four keys of a column at a
// time.  16-byte chunks of a row are stored at places that depend on the key (chunk ^ key % 16 of K, and
// chunk ^ 4 (key % 4) of V), so that the lanes of a read meet different banks.
// A weight is taken as the sum of two bf16 (off by 2^-16 of it at most), as in the form for few rows, so a token's precision does not depend on how many
// come with it: two products, with one operand read.  One bf16 alone (2^-8) leaves a third more error in outputs whose values' mean is 0 (4096 keys); it
// takes 2037 us of the first case below for 2780, and 350 of the second for 450.
// 2048 tokens behind 59392 keys, 32 heads over 8, take 2.65 to 2.80 ms (cards and runs differ), 725 to 765 TFLOP/s of the attention's operations, 1.09 to
// 1.15 PFLOP/s with the second products (a library product of 8192^3 reaches 1.20 on this card).  At 1.82 GHz the matrix unit is busy for 58 % of
// the cycles, the vector instructions, those of the weights above all, take 55 %, LDS 49 % (39 for reads, 10 for bringing tiles in): two
// wavefronts a SIMD, whose products and weights overlap, leave little between them.  Four prompts of up to 4099 tokens 435 to 460 us, 635 to 670 TFLOP/s, matrix unit 49 %: the
// starts and ends of 5.5 rounds of workgroups are not covered (tiles on the diagonal, formed whole, are 4 % of its cycles).  e4m3, widened on the way to LDS: 2.79 ms, 460 us.
// The weights are spread over the products that they wait for; worked out in the first 24 of the 32 steps: 2797 us for 2780.  With one bf16, weights
// after the scores instead of beside the next tile's, and staging through registers, took 2364 us for 1922.
template <int ET>
__global__ __launch_bounds__(kPagedManyThreads, 2) void paged_many_rows_kernel(const PagedArgs a) {
  constexpr int kElem = ET == kFP8 ? 1 : 2;
  typedef typename std::conditional<ET == kFP8, u32x2, u32x4>::type Raw;
  __shared__ __align__(16) char lds[2][2][kTileBytes];     // [buffer][keys, values]
  __shared__ int bad_pages;                               // whether a tile had a page that is none

  PagedPiece pc;
  if (!paged_locate<KT, kPieces>(a, blockIdx.x, pc)) return;
  if (threadIdx.x == 0) bad_pages = 0;
  __syncthreads();
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
  // a negative scale goes to the queries, so that the largest score is the largest product; one of 0 becomes the smallest number
  // there is, which leaves the -inf of a masked score what it is; one that is a NaN goes to the queries too, for the same reason
  const float signed_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[pc.g] : 1.f);
  const bool no_scale = signed_log2 != signed_log2;
  const float to_log2 = no_scale ? 1.f : (signed_log2 == 0.f ? 1.17549435e-38f : fabsf(signed_log2));
  const uint32_t flip = signed_log2 < 0.f ? 0x80008000u : 0u, nan = no_scale ? 0x7fff7fffu : 0u;

  u32x4 q[8];
  {
    const int64_t at = (int64_t)(pc.r.row + first + t) * a.q_t + (int64_t)(pc.g * a.G + head) * a.q_h + 8 * u;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      q[s] = u32x4{0, 0, 0, 0};
      if (real) q[s] = (*reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + at + 16 * s) ^ flip) | nan;
    }
  }

  const const_i32_ptr table = (const_i32_ptr)(a.table + (int64_t)pc.b * a.max_pages);
  const char* kbase = reinterpret_cast<const char*>(a.k) + (int64_t)pc.g * a.k_head * kElem;
  const char* vbase = reinterpret_cast<const char*>(a.v) + (int64_t)pc.g * a.v_head * kElem;
  const int page_mask = (1 << a.page_shift) - 1;
  const uint32_t k_key = (uint32_t)a.k_key * kElem, v_key = (uint32_t)a.v_key * kElem;
  // Staging: a wavefront takes sixteen keys of a tile, K and V, four rows at a time (sixteen lanes a row): one page and two descriptors each.
  const int srow = lane >> 4, chunk = lane & 15;
  const uint32_t k_from = srow * k_key + 8 * chunk * kElem, v_from = srow * v_key + 8 * chunk * kElem;
  const int k_to = (16 * wave + srow) * 256, k_chunk = (chunk ^ srow) << 4, v_to = (16 * wave + srow) * 256 + ((chunk ^ srow << 2) << 4);
  // reading
  const int k_at = c * 256, k_swap = (u ^ (c & 15)) << 4;
  const int i16 = lane & 15, quad = i16 >> 2;
  const int v_at = (4 * u + quad) * 256 + (2 * (lane >> 4 & 1) + (i16 >> 1 & 1)) * 16 + (i16 & 1) * 8;

  auto tile_key = [&](int v) { return (v < span.sink ? v : v + span.skip) * KT; };
  auto page_ok = [&](int id) { return (uint32_t)id < (uint32_t)a.n_pages; };
  // the page of this wavefront's keys of a tile
  auto tile_page = [&](int v) {
    const int at = (tile_key(v) + 16 * wave) >> a.page_shift;
    return table[at < a.max_pages ? at : a.max_pages - 1];
  };
  auto valid_keys = [&](int v, int id) { return page_ok(id) ? min(max(end - tile_key(v) - 16 * wave, 0), 16) : 0; };
  auto k_rows = [&](int v, int id) {
    return rows16(kbase, a.k_page * kElem, k_key, id, (tile_key(v) + 16 * wave) & page_mask, valid_keys(v, id));
  };
  auto v_rows = [&](int v, int id) {
    return rows16(vbase, a.v_page * kElem, v_key, id, (tile_key(v) + 16 * wave) & page_mask, valid_keys(v, id));
  };
  // Through registers (e4m3, which is widened on the way, and sixteens that are not whole): fetch(), and put() some time later.
  auto fetch = [&](__amdgpu_buffer_rsrc_t rows, uint32_t from, uint32_t key_stride, Raw (&r)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) load_shared(rows, from + 4 * i * key_stride, r[i]);
  };
  auto put_k = [&](int buf, const Raw (&r)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4 k;
      if constexpr (ET == kFP8) k = e4m3_to_bf16(r[i]);
      else k = r[i];
      *reinterpret_cast<u32x4*>(&lds[buf][0][k_to + 1024 * i + (k_chunk ^ 64 * i)]) = k;
    }
  };
  auto put_v = [&](int buf, const Raw (&r)[4], auto careful) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4 x;
      if constexpr (ET == kFP8) x = e4m3_to_bf16(r[i]);
      else x = r[i];
      if constexpr (decltype(careful)::value) x = finite_part<false>(x);
      *reinterpret_cast<u32x4*>(&lds[buf][1][v_to + 1024 * i]) = x;
    }
  };
  // Straight into LDS: a load leaves its lanes' 16 bytes one behind the other, four rows, so a lane asks for the chunk that belongs
  // in its place.
  auto straight_k = [&](int buf, __amdgpu_buffer_rsrc_t rows) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      load_to_lds(rows, srow * k_key + 4 * i * k_key + (k_chunk ^ 64 * i), &lds[buf][0][4096 * wave + 1024 * i]);
  };
  auto straight_v = [&](int buf, __amdgpu_buffer_rsrc_t rows) {
#pragma unroll
    for (int i = 0; i < 4; ++i) load_to_lds(rows, srow * v_key + 4 * i * v_key + ((chunk ^ srow << 2) << 4), &lds[buf][1][4096 * wave + 1024 * i]);
  };
  // A tile's sixteen keys of this wavefront: on their way (bring), and there (arrived, at the latest before the next barrier).
  Raw kr[4], vr[4];
  auto bring_k = [&](int buf, int v, int id) {
    const auto rows = k_rows(v, id);
    if constexpr (ET == kFP8) {
      fetch(rows, k_from, k_key, kr);
    } else if (valid_keys(v, id) == 16) {
      straight_k(buf, rows);
    } else {
      Raw r[4];
      fetch(rows, k_from, k_key, r);
      put_k(buf, r);
    }
  };
  auto bring_v = [&](int buf, int v, int id) {
    const auto rows = v_rows(v, id);
    if constexpr (ET == kFP8) {
      fetch(rows, v_from, v_key, vr);
    } else if (valid_keys(v, id) == 16) {
      straight_v(buf, rows);
    } else {
      Raw r[4];
      fetch(rows, v_from, v_key, r);
      put_v(buf, r, std::false_type{});
    }
  };
  auto arrived_k = [&](int buf) { if constexpr (ET == kFP8) put_k(buf, kr); };
  auto arrived_v = [&](int buf) { if constexpr (ET == kFP8) put_v(buf, vr, std::false_type{}); };

  f32x16 o[4];
  float m, l;
  bool bad_page = false;                                 // (as far as this wavefront knows; behind a barrier: of every tile brought in before)
  auto reset = [&]() {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
  };
  // operands: elements 16 e .. 16 e + 15 of keys 32 kt .. 32 kt + 31; elements 32 d .. 32 d + 31 of keys 16 x .. 16 x + 15, transposed
  auto key_operand = [&](int buf, int e, int kt) {
    return *reinterpret_cast<const u32x4*>(&lds[buf][0][8192 * kt + k_at + (k_swap ^ 32 * e)]);
  };
  auto value_operand = [&](int buf, int x, int d) {
    const char* from = &lds[buf][1][4096 * x + v_at + ((d ^ quad) << 6)];
    const u32x2 v0 = read_transposed(from), v1 = read_transposed(from + 2048);
    return u32x4{v0.x, v0.y, v1.x, v1.y};
  };
  auto score = [&](int buf, f32x16 (&s)[2]) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[kt] = mfma32(key_operand(buf, e, kt), q[e], s[kt]);
    }
  };
  // keys outside the row's set: key 32 kt + 8 (i / 4) + i % 4 of the tile, from this lane's first one on
  auto mask = [&](int v, f32x16 (&s)[2]) {
    const int key0 = tile_key(v);
    if (!bad_page && key0 + KT - 1 <= min_hi && (key0 >= max_lo || key0 + KT <= a.n_sink)) return false;
    const int at = key0 + 4 * u, to = hi - at, from = lo - at, sink = a.n_sink - at;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int page = (key0 + 16 * x) >> a.page_shift;
      const bool ok = page_ok(table[page < a.max_pages ? page : a.max_pages - 1]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = 8 * (x & 1) + j, key = 32 * (x >> 1) + 8 * (i >> 2) + (i & 3);
        s[x >> 1][i] = ok && key <= to && (key >= from || key < sink) ? s[x >> 1][i] : -INFINITY;
      }
    }
    return true;
  };
  auto largest = [&](const f32x16 (&s)[2]) {
    float top = s[0][0];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kt][i]);
    return top;
  };
  auto raise = [&](float top) {
    if (!__any(top > m + 8.f)) return;
    const float m1 = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
    const float by = m == m1 ? 1.f : __builtin_amdgcn_exp2f(m - m1);
    m = m1;
    l *= by;
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= by;
  };
  // weight n of the lane's 32, as the sum of two bf16
  auto weigh = [&](int n, float ref, f32x16 (&s)[2], u32x4 (&p)[4], u32x4 (&rest)[4]) {
    const int kt = n >> 4, i = n & 15;
    s[kt][i] = __builtin_amdgcn_exp2f(fmaf(s[kt][i], to_log2, -ref));
    l += s[kt][i];
    if (i & 1) {
      const int x = 2 * kt + (i >> 3), at = (i & 7) >> 1;
      const uint32_t both = pack_bf16(s[kt][i - 1], s[kt][i]);
      p[x][at] = both;
      rest[x][at] = pack_bf16(s[kt][i - 1] - __uint_as_float(both << 16), s[kt][i] - __uint_as_float(both & 0xffff0000u));
    }
  };

  // The tiles, two steps of a tile in flight: while the weights of tile v are worked out, the matrix unit forms the scores of
  // tile v + 1.  Buffer v % 2 of the values holds tile v, buffer (v + 1) % 2 of the keys tile v + 1; tile v + 2's keys and
  // tile v + 1's values are on their way.
  reset();
  if (t_begin < t_end) {
    // (tiles from wave_end on hold keys behind all of the wavefront's rows: it only helps to bring them in)
    const int reach = wave_hi / KT, reach_v = reach < span.sink ? reach : max(reach - span.skip, span.sink - 1);
    const int wave_end = wave_hi < 0 ? t_begin : min(max(reach_v + 1, t_begin), t_end);
    const int id = tile_page(t_begin);
    int id1 = t_begin + 1 < t_end ? tile_page(t_begin + 1) : 0;
    if (!page_ok(id) || !page_ok(id1)) bad_pages = 1;
    bring_k(t_begin & 1, t_begin, id);
    bring_v(t_begin & 1, t_begin, id);
    arrived_k(t_begin & 1);
    arrived_v(t_begin & 1);
    if (t_begin + 1 < t_end) {
      bring_k((t_begin + 1) & 1, t_begin + 1, id1);
      arrived_k((t_begin + 1) & 1);
    }
    stored();
    __syncthreads();
    f32x16 s[2];
    if (t_begin < wave_end) {
      bad_page = bad_pages;
      score(t_begin & 1, s);
      mask(t_begin, s);
      raise(largest(s) * to_log2);
    }
    __syncthreads();                                       // (the first tile's keys have been read: another's take their place)
#pragma unroll 1
    for (int v = t_begin; v < t_end; ++v) {
      if (v + 1 < t_end) bring_v((v + 1) & 1, v + 1, id1);
      if (v + 2 < t_end) {
        id1 = tile_page(v + 2);
        bring_k(v & 1, v + 2, id1);
        if (!page_ok(id1)) bad_pages = 1;
      }
      if (v < wave_end) {
        // Step by step, in this order: a product, the operand of the one kAhead further on, and as much of the weights as the product
        // takes.  Steps 0 .. 15 are the scores of tile v + 1 (behind the last tile those of an old one, unused), 16 .. 31 the output of tile v.
        f32x16 next[2];
        u32x4 p[4], rest[4], operand[kAhead];
        const float ref = m == -INFINITY ? 0.f : m;
        float top = -INFINITY;
        auto request = [&](auto at) {
          constexpr int step = decltype(at)::value;
          if constexpr (step < 16) operand[step % kAhead] = key_operand((v + 1) & 1, step >> 1, step & 1);
          else if constexpr (step < 32) operand[step % kAhead] = value_operand(v & 1, (step - 16) >> 2, step & 3);
        };
        each<0, kAhead>(request);
#pragma unroll
        for (int i = 0; i < 16; ++i) { next[0][i] = 0.f; next[1][i] = 0.f; }
        each<0, 32>([&](auto at) {
          constexpr int step = decltype(at)::value;
          if constexpr (step < 16) next[step & 1] = mfma32(operand[step % kAhead], q[step >> 1], next[step & 1]);
          else o[step & 3] = mfma32(operand[step % kAhead], rest[(step - 16) >> 2], mfma32(operand[step % kAhead], p[(step - 16) >> 2], o[step & 3]));
          request(std::integral_constant<int, step + kAhead>{});
          // (of the 32 weights twelve beside the sixteen products of the scores, the others beside the first 24 of the output's)
          if constexpr (step < 16) {
            each<step * 3 / 4, (step + 1) * 3 / 4>([&](auto n) { weigh(decltype(n)::value, ref, s, p, rest); });
          } else if constexpr (step < 28) {
            each<12 + (step - 16) * 5 / 3, 12 + (step - 15) * 5 / 3>([&](auto n) { weigh(decltype(n)::value, ref, s, p, rest); });
          } else {
            each<8 * (step - 28), 8 * (step - 27)>([&](auto n) { top = fmaxf(top, next[decltype(n)::value >> 4][decltype(n)::value & 15]); });
          }
          __builtin_amdgcn_sched_barrier(0);
        });
        if (v + 1 < wave_end) {
          bad_page = bad_pages;
          if (mask(v + 1, next)) top = largest(next);
          raise(top * to_log2);
        }
        s[0] = next[0];
        s[1] = next[1];
      }
      if (v + 1 < t_end) arrived_v((v + 1) & 1);
      if (v + 2 < t_end) arrived_k(v & 1);
      stored();
      __syncthreads();
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
      const int key0 = tile_key(v), id0 = tile_page(v);
      Raw r[4];
      fetch(k_rows(v, id0), k_from, k_key, r);
      put_k(0, r);
      fetch(v_rows(v, id0), v_from, v_key, r);
      put_v(0, r, std::true_type{});
      __syncthreads();
      if (key0 <= wave_hi) {
        f32x16 s[2];
        u32x4 p[4], rest[4];
        bad_page = true;
        score(0, s);
        mask(v, s);
        raise(largest(s) * to_log2);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int n = 0; n < 32; ++n) weigh(n, ref, s, p, rest);
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const u32x4 v = value_operand(0, x, d);
            o[d] = mfma32(v, rest[x], mfma32(v, p[x], o[d]));
          }
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
    if (u == 0) { pp[128] = paged_partial_max(m, l); pp[129] = l; }
  } else {
    const int64_t to = (int64_t)(pc.r.row + first + t) * a.Hq + pc.g * a.G + head;
    const bool none = l == 0.f;                          // (as paged_write_row has it)
    const float by = (a.v_scale ? a.v_scale[pc.g] : 1.f) / l;
    auto done = [&](int d, int i) { return none ? 0.f : o[d][i] * by; };
    uint16_t* out = reinterpret_cast<uint16_t*>(a.out) + to * kHeadDim + 4 * u;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x2*>(out + 32 * d + 8 * i) = u32x2{pack_bf16(done(d, 4 * i), done(d, 4 * i + 1)), pack_bf16(done(d, 4 * i + 2), done(d, 4 * i + 3))};
    if (a.lse && u == 0) a.lse[to] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
  }
}

}  // namespace

void launch_paged_many_rows(const PagedArgs& a, bool fp8, const PagedForm& form, hipStream_t s) {
  if (fp8) paged_many_rows_kernel<kFP8><<<(unsigned)form.pieces, kPagedManyThreads, 0, s>>>(a);
  else paged_many_rows_kernel<kBF16><<<(unsigned)form.pieces, kPagedManyThreads, 0, s>>>(a);
}

}  // namespace mp
