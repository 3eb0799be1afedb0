// What the step's attention weighs each cached key with, added to the key's account.
#include "paged_device.h"

#include <type_traits>

namespace mp {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;

// Few rows: keys of a tile, and loads of a lane for sixteen of them.
template <int ET, int NR = 1>
struct Tile {
  static constexpr int kKeys = weights_tile(ET == kFP32, ET == kBF16 ? 16 : 8, 16 * NR);
  static constexpr int kHalves = kKeys / 16;
  static constexpr int kFrags = ET == kFP32 ? 8 : (ET == kBF16 ? 4 : (ET == kFP8 ? 2 : 1));
  static constexpr int kValues = 4 * kHalves;              // scores of a lane: key 16 (i / 4) + 4 u + i % 4 is number i
};

// The tiles of a request that are looked at: those of the sink, then those from the window of the first new token on, or from the first key
// without an account.  Tile v is tile v of the cache, or v + skip from `sink` on.
struct Reach {
  int len, tokens, row, counted, tiles, sink, skip;
};
__device__ inline Reach reach_of(const PageWeightsArgs& a, int b, int KT) {
  const PagedRequest r = paged_request(a.paged, b);
  Reach x{r.len, r.tokens, r.row, 0, 0, 0, 0};
  const int old = r.len - r.tokens;                        // (below 0 where there are more new tokens than keys)
  int counted = a.counted ? a.counted[b] : old;
  x.counted = counted < 0 ? 0 : (counted > r.len ? r.len : counted);
  int from = 0, sink = 0;
  if (r.tokens == 0) {
    from = x.counted;
  } else if (a.paged.n_local > 0) {
    const int lo = old - a.paged.n_local + 1;
    from = lo < x.counted ? lo : x.counted;
    from = from < 0 ? 0 : from;
    sink = a.paged.n_sink < from ? a.paged.n_sink : from;
  }
  x.sink = (sink + KT - 1) / KT;
  x.skip = from / KT - x.sink;
  if (x.skip < 0) x.skip = 0;
  x.tiles = (r.len + KT - 1) / KT - x.skip;
  if (from >= r.len && sink == 0) x.tiles = 0;
  return x;
}

// The lane's place among sixteen keys and their elements.
struct Place {
  int lane, c, u, quad, in_quad;
  __device__ Place() : lane(threadIdx.x & 63), c(lane & 15), u(lane >> 4), quad(c >> 2), in_quad(c & 3) {}
};

// A KV head's keys.
template <int ET>
struct Keys {
  const char* base; const char* blocks;
  int64_t page, block_page;
  uint32_t key, block_key;
  __device__ Keys(const PagedArgs& a, int g)
      : base(reinterpret_cast<const char*>(a.k) + pool_bytes<ET>((int64_t)g * a.k_head)),
        blocks(reinterpret_cast<const char*>(a.k_block) + ((int64_t)g * a.k_head >> 5)), page(pool_bytes<ET>(a.k_page)), block_page(a.k_page >> 5),
        key((uint32_t)pool_bytes<ET>(a.k_key)), block_key((uint32_t)(a.k_key >> 5)) {}
};

// A tile's keys: on their way, and then as the A operand of S^T = K Q^T - lane (c, u) has elements 32 u .. 32 u + 31 of key c (float32: 16 u .. and 64 + 16 u ..).
template <int ET, int H = Tile<ET>::kHalves>
struct Operand {
  u32x4 k[H][Tile<ET>::kFrags];
  uint32_t scale[ET == kFP4 ? H : 1];

  // `valid` of sixteen keys from `at` of page id on
  __device__ inline void request(const Keys<ET>& keys, const Place& p, int h, int id, int at, int valid) {
    const auto rows = rows16(keys.base, keys.page, keys.key, id, at, valid);
    if constexpr (ET == kFP4) {
      load_shared(rows, (p.lane >> 2) * keys.key + 16 * (p.in_quad ^ p.u), k[h][0]);   // (neighbouring heads' rows share lines)
      scale[h] = load_byte(rows16(keys.blocks, keys.block_page, keys.block_key, id, at, valid), p.c * keys.block_key + p.u);
    } else if constexpr (ET == kFP8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) load_once(rows, (4 * p.quad + (p.in_quad >> 1) + 2 * i) * keys.key + 32 * p.u + 16 * (p.in_quad & 1), k[h][i]);
    } else {
#pragma unroll
      for (int i = 0; i < Tile<ET>::kFrags; ++i) load_once(rows, (4 * p.quad + (i & 3)) * keys.key + 64 * p.u + 16 * p.in_quad + 256 * (i >> 2), k[h][i]);
    }
  }
  // Lanes exchange what they loaded; `lds`: 4096 bytes of the wavefront's own (four bits).
  __device__ inline void arrange(const Place& p, char* lds) {
    if constexpr (ET == kFP4) {
#pragma unroll
      for (int h0 = 0; h0 < H; h0 += 4) {
#pragma unroll
        for (int h = h0; h < h0 + 4 && h < H; ++h) *reinterpret_cast<u32x4*>(lds + 1024 * (h - h0) + 16 * p.lane) = k[h][0];
        in_order();
#pragma unroll
        for (int h = h0; h < h0 + 4 && h < H; ++h) k[h][0] = *reinterpret_cast<const u32x4*>(lds + 1024 * (h - h0) + 64 * p.c + 16 * (p.u ^ p.quad));
        in_order();
      }
    } else {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if constexpr (ET == kFP8) join_halves(k[h][0], k[h][1], p.c & 2);
        else
#pragma unroll
          for (int x = 0; x < Tile<ET>::kFrags; x += 4) transpose_quads(k[h][x], k[h][x + 1], k[h][x + 2], k[h][x + 3], p.c & 1, p.c & 2);
      }
    }
  }
  // elements 32 u + 8 i .. of half h as bf16
  __device__ inline u32x4 bf16(int h, int i) const {
    if constexpr (ET == kFP4) return e2m1_to_bf16(k[h][0][i], scale[h] << 23);
    else if constexpr (ET == kFP8) return e4m3_to_bf16(i & 1 ? u32x2{k[h][i >> 1].z, k[h][i >> 1].w} : u32x2{k[h][i >> 1].x, k[h][i >> 1].y});
    else return k[h][i];
  }
};

constexpr int q_frags(int et) { return et == kFP32 ? 8 : 4; }

// One query row as the B operand, from global memory.
template <int ET>
__device__ inline void load_query(const PagedArgs& a, int64_t at, const Place& p, bool real, u32x4 (&q)[q_frags(ET)]) {
#pragma unroll
  for (int s = 0; s < q_frags(ET); ++s) {
    q[s] = u32x4{0, 0, 0, 0};
    const int e = ET == kFP32 ? 64 * (s >> 2) + 16 * p.u + 4 * (s & 3) : 32 * p.u + 8 * s;
    if (real) {
      if constexpr (ET == kFP32) q[s] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(a.q) + at + e);
      else q[s] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(a.q) + at + e);
    }
  }
}

// Scores of half h with sixteen rows.
template <int ET, int H>
__device__ inline f32x4 scores(const Operand<ET, H>& k, int h, const u32x4 (&q)[q_frags(ET)]) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if constexpr (ET == kFP32) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k.k[h][i][e]), __uint_as_float(q[i][e]), s, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) s = mfma_bf16(k.bf16(h, i), q[i], s);
  }
  return s;
}

template <int CTRL>
__device__ inline float moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// Sums over the sixteen lanes c of each of N values; lane c gets that of value c % N.
template <int N>
__device__ inline float sum_rows(float (&v)[N], const Place& p) {
  constexpr int kMirror = 0x140, kHalfMirror = 0x141;      // lanes c ^ 15, c ^ 7
  // (of the lanes that are added up each keeps the half of the values that its own number says)
  if constexpr (N == 16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float m0 = moved<kMirror>(v[i]), m1 = moved<kMirror>(v[8 + i]);
      v[i] = p.c & 8 ? v[8 + i] + m1 : v[i] + m0;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += moved<kMirror>(v[i]);
  }
  if constexpr (N >= 8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float m0 = moved<kHalfMirror>(v[i]), m1 = moved<kHalfMirror>(v[4 + i]);
      v[i] = p.c & 4 ? v[4 + i] + m1 : v[i] + m0;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += moved<kHalfMirror>(v[i]);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float m0 = moved<0x4e>(v[i]), m1 = moved<0x4e>(v[2 + i]);
    v[i] = p.c & 2 ? v[2 + i] + m1 : v[i] + m0;
  }
  const float m0 = moved<0xb1>(v[0]), m1 = moved<0xb1>(v[1]);
  return p.c & 1 ? v[1] + m1 : v[0] + m0;
}

__device__ inline bool page_ok(const PagedArgs& a, int id) { return (uint32_t)id < (uint32_t)a.n_pages; }

template <int H>
__device__ inline void tile_pages(const PagedArgs& a, const_i32_ptr table, int key0, int (&id)[H]) {
#pragma unroll
  for (int h = 0; h < H; ++h) {
    const int at = (key0 + 16 * h) >> a.page_shift;
    id[h] = table[at < a.max_pages ? at : a.max_pages - 1];
  }
}
template <int ET, int H>
__device__ inline void request_tile(const PagedArgs& a, const Keys<ET>& keys, const Place& p, int key0, int end, const int (&id)[H], Operand<ET, H>& k) {
  const int page_mask = (1 << a.page_shift) - 1;
#pragma unroll
  for (int h = 0; h < H; ++h)
    k.request(keys, p, h, id[h], (key0 + 16 * h) & page_mask, page_ok(a, id[h]) ? min(max(end - key0 - 16 * h, 0), 16) : 0);
}
// Where the account of the lane's key is, key 16 (v / 4) + 4 u + v % 4 of the tile for v = c % (4 halves); null where it has none, or another lane has it.
template <int H>
__device__ inline float* account(const PageWeightsArgs& a, const Place& p, int g, int key0, int len, const int (&id)[H], int& key) {
  key = key0 + 16 * (p.quad & (H - 1)) + 4 * p.u + p.in_quad;
  int page = id[0];
#pragma unroll
  for (int h = 1; h < H; ++h) page = (p.quad & (H - 1)) == h ? id[h] : page;
  if (p.c >= 4 * H || key >= len || !page_ok(a.paged, page)) return nullptr;
  return a.weights + ((((int64_t)page * a.paged.Hkv + g) << a.paged.page_shift) + (key & ((1 << a.paged.page_shift) - 1)));
}

// ---- few rows: a wavefront has all of a request's rows of a KV head -----------------------------------
// Scores are formed as S^T = K Q^T, so a lane has four keys of a query row (column c) in each MFMA: a weight is exp2(score - lse), no maximum and no sum have to be
// known first, and a key's sum over the rows is one over registers and sixteen lanes.  Every key of a request belongs to one wavefront: no atomics, and the same bits
// every time (a page that two requests name is added to by two: its accounts are not defined).  The log-sum-exp is taken to base 2 in float32, which moves a row's weights by about
// 2^-24 |lse| of themselves at most, as a rounding of lse itself would; a second term would cost an instruction for every weight.  Workgroups take equal, contiguous shares of all tiles; the wavefronts of one take `heads` neighbouring KV heads, whose rows lie side by side in
// many pools, and waves / heads tiles at a time.  Bound by memory: 16 requests of 32768 keys, four rows (bf16, 1.11 GB) 194 us, 5.7 TB/s; 32 rows 203, 64 rows
// 215, 128 rows 376 (their exponentials); e4m3 113 to 117, four bits 74 to 79 (4.1 to 4.3 TB/s: widening), float32, 8 requests, 182 to 184, 5.9 TB/s.  64 rows by the form for many 476, 128 rows 862 (its rows then split among wavefronts).
template <int ET, int NR>
__global__ __launch_bounds__(kThreads, NR <= 2 ? 4 : 2) void page_weights_few_kernel(const PageWeightsArgs w) {
  using T = Tile<ET, NR>;
  constexpr int KT = T::kKeys, kTogether = NR < 2 ? NR : 2;   // rows (sixteens of them) whose scores are there at once
  __shared__ __align__(16) char lds[ET == kFP4 ? kWaves * 4096 : 16];
  const PagedArgs& a = w.paged;
  const Place p;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at_once = kWaves / w.heads, head = wave % w.heads, place = wave / w.heads, sets = a.Hkv / w.heads;
  auto groups_of = [&](int b) { return (reach_of(w, b, KT).tiles + at_once - 1) / at_once * sets; };
  int total = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) total += __builtin_amdgcn_readlane(wave_prefix(b0 + p.lane < a.batch ? groups_of(b0 + p.lane) : 0), 63);
  const int each = (total + gridDim.x - 1) / gridDim.x;
  int pos = each * blockIdx.x;
  const int end = min(pos + each, total);
  if (pos >= end) return;
  int b = 0, base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int n = b0 + p.lane < a.batch ? groups_of(b0 + p.lane) : 0, upto = wave_prefix(n);
    const uint64_t found = __ballot(base + upto > pos);
    if (found) {
      const int f = __ffsll((unsigned long long)found) - 1;
      b = b0 + f;
      base += __builtin_amdgcn_readlane(upto - n, f);
      break;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
#pragma unroll 1
  while (pos < end) {
    b = __builtin_amdgcn_readfirstlane(b);
    const Reach x = reach_of(w, b, KT);
    const int groups = (x.tiles + at_once - 1) / at_once;
    if (groups * sets <= pos - base) {                     // (requests without tiles)
      base += groups * sets;
      ++b;
      continue;
    }
    const int set = (pos - base) / groups, from = pos - base - set * groups, to = min(groups, from + end - pos);
    pos += to - from;
    const int g = set * w.heads + head;
    // this lane's rows
    u32x4 q[NR][q_frags(ET)];
    float lse[NR];
    int hi[NR], lo[NR];
    const int rows = x.tokens * a.G;
    bool counts = true;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int row = p.c + 16 * n, t = row / a.G, h = row - t * a.G;
      bool real = row < rows;
      lse[n] = INFINITY;
      if (real) lse[n] = w.lse[(int64_t)(x.row + t) * a.Hq + g * a.G + h] * 1.4426950408889634f;
      real = real && lse[n] != -INFINITY;                  // (a row that attends nothing)
      counts = counts && real;
      hi[n] = real ? x.len - x.tokens + t : -1;
      lo[n] = a.n_local > 0 ? hi[n] - a.n_local + 1 : 0;
      load_query<ET>(a, (int64_t)(x.row + t) * a.q_t + (int64_t)(g * a.G + h) * a.q_h, p, real, q[n]);
    }
    const bool all = __all(counts);                        // whether every lane has rows that count
    const int min_hi = x.len - x.tokens, max_lo = a.n_local > 0 ? x.len - a.n_local : 0;
    const float to_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[g] : 1.f);
    const Keys<ET> keys(a, g);
    const const_i32_ptr table = (const_i32_ptr)(a.table + (int64_t)b * a.max_pages);
    char* const mine = lds + (ET == kFP4 ? 4096 * wave : 0);
    auto tile_key = [&](int v) { return (v < x.sink ? v : v + x.skip) * KT; };
    int v = from * at_once + place;
    const int v_end = min(to * at_once, x.tiles);
    Operand<ET, T::kHalves> k;
    int id[T::kHalves], key = 0;
    float* to_account = nullptr;
    float old = 0.f;
    auto bring = [&](int v) {
      const int key0 = tile_key(v);
      tile_pages<T::kHalves>(a, table, key0, id);
      request_tile<ET, T::kHalves>(a, keys, p, key0, x.len, id, k);
      to_account = account(w, p, g, key0, x.len, id, key);
      old = to_account && key < x.counted ? *to_account : 0.f;
    };
    if (v < v_end) bring(v);
#pragma unroll 1
    while (v < v_end) {
      const int key0 = tile_key(v);
      k.arrange(p, mine);
      float s[T::kValues];
#pragma unroll
      for (int i = 0; i < T::kValues; ++i) s[i] = 0.f;
      float part[kTogether][T::kValues];
      const bool full = key0 + KT - 1 <= min_hi && (key0 >= max_lo || key0 + KT <= a.n_sink);
      float* const to_now = to_account;
      const float old_now = old;
      v += at_once;
#pragma unroll
      for (int n0 = 0; n0 < NR; n0 += kTogether) {
#pragma unroll
        for (int n = 0; n < kTogether; ++n)
#pragma unroll
          for (int h = 0; h < T::kHalves; ++h) {
            const f32x4 x4 = scores(k, h, q[n0 + n]);
#pragma unroll
            for (int i = 0; i < 4; ++i) part[n][4 * h + i] = x4[i];
          }
        if (n0 + kTogether == NR && v < v_end) bring(v);
#pragma unroll
        for (int n = 0; n < kTogether; ++n)
#pragma unroll
          for (int i = 0; i < T::kValues; ++i) {
            float e = __builtin_amdgcn_exp2f(fmaf(part[n][i], to_log2, -lse[n0 + n]));
            if (!full) {
              const int at = key0 + 16 * (i >> 2) + 4 * p.u + (i & 3);
              e = at <= hi[n0 + n] && (at >= lo[n0 + n] || at < a.n_sink) ? e : 0.f;
            } else if (!all) {
              e = hi[n0 + n] >= 0 ? e : 0.f;               // (the position of a row that counts is min_hi or more)
            }
            s[i] += e;
          }
      }
      const float add = sum_rows<T::kValues>(s, p);
      if (to_now) *to_now = old_now + add;
    }
    if (set + 1 == sets && to == groups) {
      base += groups * sets;
      ++b;
    }
  }
}

// ---- many rows: a wavefront has a tile of 64 keys and goes over its share of the rows ---------------------
// The keys stay in registers as bf16 (float32: 32 keys as they are), the rows come by: 32 at a time, loaded with neighbouring lanes on neighbouring addresses and
// handed over in the wavefront's part of LDS, the next ones on their way.  The wavefronts of a workgroup are `row_split` shares of the rows, of one tile or of several.
// Bound by the exponentials' and the products' cycles where there are many keys (2048 tokens behind 59392 keys, 32 heads over 8: 1.36 ms, 0.75 PFLOP/s) and by
// the way of the rows from L2 and the wavefronts' ends where there are few: four prompts of up to 4099 tokens 251 to 294 us, 0.5 to 0.58 PFLOP/s (e4m3 260, four bits 262, float32 1490; 40 heads over 8, whose tokens steps of rows end in, 380), matrix unit 26 % busy before
// rows came 32 at a time.  Rows loaded as operands, 64 addresses a load: 660 us; 96 and 128 keys a wavefront: registers spill, and every reload waits for the
// rows on their way, 640 and 1160.
template <int ET>
struct Many {
  static constexpr bool kF32 = ET == kFP32;
  static constexpr int kHalves = kF32 ? 2 : 4, kKeys = 16 * kHalves, kFrags = q_frags(ET), kValues = 4 * kHalves;
  static constexpr int kTiles = 2, kRows = 16 * kTiles;  // query rows that come by at once
  static constexpr int kRowBytes = kF32 ? 512 : 256, kPerLoad = 1024 / kRowBytes, kLoads = kRows / kPerLoad;   // of a row; rows of a load of the wavefront
};

template <int ET>
__global__ __launch_bounds__(64 * kWeightsManyWaves, 2) void page_weights_many_kernel(const PageWeightsArgs w) {
  using M = Many<ET>;
  constexpr int kWaves = kWeightsManyWaves, kThreads = 64 * kWaves;
  __shared__ __align__(16) char lds[kWaves][M::kRows * M::kRowBytes];
  __shared__ float sums[kWaves][M::kKeys];
  const PagedArgs& a = w.paged;
  const Place p;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row_split = w.heads, tile_of = wave / row_split, share = wave % row_split, block = kWaves / row_split * M::kKeys;
  char* const mine = lds[wave];
#pragma unroll 1
  for (int64_t index = blockIdx.x;; index += gridDim.x) {
    // item: KV head, block of keys, request
    const int g = (int)(index % a.Hkv);
    int64_t rest = index / a.Hkv;
    int b = -1;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      const int n = b0 + p.lane < a.batch ? reach_of(w, b0 + p.lane, block).tiles : 0, upto = wave_prefix(n);
      const uint64_t found = __ballot(upto > rest);
      if (found) {
        const int f = __ffsll((unsigned long long)found) - 1;
        b = b0 + f;
        rest -= __builtin_amdgcn_readlane(upto - n, f);
        break;
      }
      rest -= __builtin_amdgcn_readlane(upto, 63);
    }
    if (b < 0) return;
    b = __builtin_amdgcn_readfirstlane(b);
    const Reach x = reach_of(w, b, block);
    const int v = __builtin_amdgcn_readfirstlane((int)rest), block0 = (v < x.sink ? v : v + x.skip) * block, key0 = block0 + tile_of * M::kKeys;
    const float to_log2 = a.scale_log2 * (a.k_scale ? a.k_scale[g] : 1.f);
    const const_i32_ptr table = (const_i32_ptr)(a.table + (int64_t)b * a.max_pages);
    u32x4 k[M::kHalves][M::kFrags];
    {
      const Keys<ET> keys(a, g);
      Operand<ET, M::kHalves> raw;
      int id[M::kHalves];
      tile_pages<M::kHalves>(a, table, key0, id);
      request_tile<ET, M::kHalves>(a, keys, p, key0, x.len, id, raw);
      raw.arrange(p, mine);
#pragma unroll
      for (int h = 0; h < M::kHalves; ++h)
#pragma unroll
        for (int i = 0; i < M::kFrags; ++i) {
          if constexpr (M::kF32) k[h][i] = raw.k[h][i];
          else k[h][i] = raw.bf16(h, i);
        }
    }
    // rows of tokens that attend a key of the tile: from the first one at or behind its first key, to the last one whose window has its last key
    const int old = x.len - x.tokens, rows = x.tokens * a.G;
    int t_end = x.tokens;
    if (a.n_local > 0 && key0 >= a.n_sink) t_end = (int)min((int64_t)t_end, (int64_t)key0 + M::kKeys - 1 + a.n_local - old);
    const int r_end = key0 < x.len ? max(t_end, 0) * a.G : 0, r_begin = max(key0 - old, 0) * a.G / 16 * 16 + M::kRows * share, r_step = M::kRows * row_split;
    // This lane's rows: those it loads a part of, and its column's.  They go on by r_step rows, dt tokens and dh heads.  Addresses are a pointer of the
    // wavefront's, which goes with the first row, and a lane's offset from there (see next_head).  (Multiplied out they took longer
    // than the products did; 64-bit ones for each lane took registers that kept a wavefront from the compute unit.)
    const int dt = r_step / a.G, dh = r_step - dt * a.G, t0 = r_begin / a.G;
    int first_head = r_begin - t0 * a.G;
    bool first_past = false;                               // whether the first row's head went past the last one in the step of the last fetch
    constexpr int kElem = M::kF32 ? 4 : 2, kRowLanes = 64 / M::kPerLoad;
    const int part = p.lane & (kRowLanes - 1);             // of a row's sixteen bytes, those of this lane
    const char* q_at = reinterpret_cast<const char*>(a.q) + ((x.row + (int64_t)t0) * a.q_t + (int64_t)g * a.G * a.q_h) * kElem;
    const float* lse_at = w.lse + (x.row + (int64_t)t0) * a.Hq + g * a.G;
    const int q_t = (int)a.q_t * kElem, q_h = (int)a.q_h * kElem, q_wrap = q_t - a.G * q_h;
    int from[M::kLoads], head[M::kLoads], own_t[M::kTiles], own_h[M::kTiles], lse_from[M::kTiles];
#pragma unroll
    for (int i = 0; i < M::kLoads; ++i) {
      const int row = r_begin + M::kPerLoad * i + p.lane / kRowLanes, t = row / a.G;
      head[i] = row - t * a.G;
      from[i] = (t - t0) * q_t + head[i] * q_h + 16 * part;
    }
#pragma unroll
    for (int n = 0; n < M::kTiles; ++n) {
      own_t[n] = (r_begin + 16 * n + p.c) / a.G;
      own_h[n] = r_begin + 16 * n + p.c - own_t[n] * a.G;
      lse_from[n] = (own_t[n] - t0) * a.Hq + own_h[n];
    }
    u32x4 next[M::kLoads];
    float next_lse[M::kTiles];
    auto fetch = [&](int r) {
      if (r + M::kRows <= rows) {
#pragma unroll
        for (int i = 0; i < M::kLoads; ++i) next[i] = *reinterpret_cast<const u32x4*>(q_at + from[i]);
#pragma unroll
        for (int n = 0; n < M::kTiles; ++n) next_lse[n] = lse_at[lse_from[n]];
      } else {                                             // (rows behind the last one read the tile's first)
        const int first = __builtin_amdgcn_readfirstlane(from[0]);
#pragma unroll
        for (int i = 0; i < M::kLoads; ++i) next[i] = *reinterpret_cast<const u32x4*>(q_at + (r + M::kPerLoad * i + p.lane / kRowLanes < rows ? from[i] : first));
#pragma unroll
        for (int n = 0; n < M::kTiles; ++n) next_lse[n] = r + 16 * n + p.c < rows ? lse_at[lse_from[n]] : INFINITY;
      }
      first_past = next_head(first_head, dh, a.G);
      q_at += (int64_t)dt * q_t + dh * q_h + (first_past ? q_wrap : 0);
      lse_at += (int64_t)dt * a.Hq + dh + (first_past ? a.Hq - a.G : 0);
      if (dh > 0) {
#pragma unroll
        for (int i = 0; i < M::kLoads; ++i) from[i] += offset_step(next_head(head[i], dh, a.G), first_past, q_wrap);
      }
    };
    float s[M::kValues];
#pragma unroll
    for (int i = 0; i < M::kValues; ++i) s[i] = 0.f;
    if (r_begin < r_end) fetch(r_begin);
#pragma unroll 1
    for (int r0 = r_begin; r0 < r_end; r0 += r_step) {
      // chunk e of row r lies at chunk e ^ r % 16 of its place
#pragma unroll
      for (int i = 0; i < M::kLoads; ++i) {
        const int r = M::kPerLoad * i + p.lane / kRowLanes;
        *reinterpret_cast<u32x4*>(mine + r * M::kRowBytes + (part ^ (r & 15)) * 16) = next[i];
      }
      in_order();
      float lse[M::kTiles];
      int hi[M::kTiles], lo[M::kTiles], first = 0, last = 0;
      bool real = true;
#pragma unroll
      for (int n = 0; n < M::kTiles; ++n) {
        lse[n] = next_lse[n] * 1.4426950408889634f;
        const bool counts = r0 + 16 * n + p.c < rows && lse[n] != -INFINITY;
        real = real && counts;
        hi[n] = counts ? old + own_t[n] : -1;
        lo[n] = a.n_local > 0 ? hi[n] - a.n_local + 1 : 0;
        if (n == 0) first = old + __builtin_amdgcn_readlane(own_t[n], 0);
        last = old + __builtin_amdgcn_readlane(own_t[n], 15);
        own_t[n] += dt;
        if (dh > 0) {
          const bool past = next_head(own_h[n], dh, a.G);
          own_t[n] += past ? 1 : 0;
          lse_from[n] += offset_step(past, first_past, a.Hq - a.G);
        }
      }
      if (r0 + r_step < r_end) fetch(r0 + r_step);
      const bool full = __all(real) && key0 + M::kKeys - 1 <= first && (a.n_local == 0 || key0 > last - a.n_local || key0 + M::kKeys <= a.n_sink);
      auto add = [&](int n, auto masked) {
        u32x4 q[M::kFrags];
#pragma unroll
        for (int i = 0; i < M::kFrags; ++i) {
          const int chunk = M::kF32 ? 16 * (i >> 2) + 4 * p.u + (i & 3) : 4 * p.u + i;
          q[i] = *reinterpret_cast<const u32x4*>(mine + (16 * n + p.c) * M::kRowBytes + (chunk ^ p.c) * 16);
        }
        f32x4 x4[M::kHalves];                              // (the products of different keys in turn: none waits for the one before it)
#pragma unroll
        for (int h = 0; h < M::kHalves; ++h) x4[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < M::kFrags; ++i) {
          if constexpr (M::kF32) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int h = 0; h < M::kHalves; ++h)
                x4[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[h][i][e]), __uint_as_float(q[i][e]), x4[h], 0, 0, 0);
          } else {
#pragma unroll
            for (int h = 0; h < M::kHalves; ++h) x4[h] = mfma_bf16(k[h][i], q[i], x4[h]);
          }
        }
#pragma unroll
        for (int h = 0; h < M::kHalves; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float e = __builtin_amdgcn_exp2f(fmaf(x4[h][i], to_log2, -lse[n]));
            if constexpr (decltype(masked)::value) {
              const int at = key0 + 16 * h + 4 * p.u + i;
              e = (at <= hi[n]) & ((at >= lo[n]) | (at < a.n_sink)) ? e : 0.f;
            }
            s[4 * h + i] += e;
          }
      };
      if (full) {
#pragma unroll
        for (int n = 0; n < M::kTiles; ++n) add(n, std::false_type{});
      } else {
#pragma unroll
        for (int n = 0; n < M::kTiles; ++n) add(n, std::true_type{});
      }
      in_order();
    }
    // over the rows of a wavefront, then over the wavefronts
    constexpr int kAtOnce = 8;
#pragma unroll
    for (int n = 0; n < M::kValues; n += kAtOnce) {
      float part[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) part[i] = s[n + i];
      const float add = sum_rows<kAtOnce>(part, p);
      if (p.c < kAtOnce) sums[wave][4 * n + 16 * (p.c >> 2) + 4 * p.u + (p.c & 3)] = add;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < block; i += kThreads) {
      const int key = block0 + i;
      if (key >= x.len) continue;
      const int id = table[key >> a.page_shift];
      if (!page_ok(a, id)) continue;
      float* const to = w.weights + ((((int64_t)id * a.Hkv + g) << a.page_shift) + (key & ((1 << a.page_shift) - 1)));
      float total = key < x.counted ? *to : 0.f;
      const int first = i / M::kKeys * row_split;
      for (int n = 0; n < row_split; ++n) total += sums[first + n][i % M::kKeys];
      *to = total;
    }
    __syncthreads();
  }
}

template <int ET, int NR>
void launch_few(const PageWeightsArgs& a, const WeightsForm& f, hipStream_t s) {
  page_weights_few_kernel<ET, NR><<<(unsigned)f.workgroups, kThreads, 0, s>>>(a);
}
template <int ET>
hipError_t launch(const PageWeightsArgs& a, const WeightsForm& f, hipStream_t s) {
  if (f.many) {
    page_weights_many_kernel<ET><<<(unsigned)f.workgroups, 64 * kWeightsManyWaves, 0, s>>>(a);
  } else if (f.rows == 16) {
    launch_few<ET, 1>(a, f, s);
  } else if constexpr (ET != kFP32) {                      // (sixteen rows of float32 at most)
    if (f.rows == 32) launch_few<ET, 2>(a, f, s);
    else if (f.rows == 64) launch_few<ET, 4>(a, f, s);
    else launch_few<ET, 8>(a, f, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_weights(const PageWeightsArgs& a, int element, const WeightsForm& f, hipStream_t s) {
  switch (element) {
    case kFP32: return launch<kFP32>(a, f, s);
    case kFP8: return launch<kFP8>(a, f, s);
    case kFP4: return launch<kFP4>(a, f, s);
    default: return launch<kBF16>(a, f, s);
  }
}

}  // namespace mp
