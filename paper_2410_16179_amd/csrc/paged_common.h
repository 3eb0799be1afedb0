// Launch descriptions of the paged cache's kernels, and how the work of paged attention is cut.
#pragma once
#include "mp_common.h"
#include "device_utils.h"

namespace mp {

struct PagePlanArgs {
  const int* new_tokens; const int* lengths; int* table; int* free_pages; const int* n_free;
  int* lengths_out; int* n_free_out; int* token_start; int64_t* slots; int* status;
  int* scan;              // workspace: the three prefix sums, [3][batch + 1] (the two-launch form)
  int batch, page_shift, max_pages, max_new;
  int64_t n_pages, max_tokens;
};

struct PageAppendArgs {
  const void* k_new; const void* v_new; const int64_t* slots; const float* k_scale; const float* v_scale;
  void* k_pages; void* v_pages;
  int heads, page_shift, is_fp32, kv_fp8;
  int64_t n_slots, tokens;
  int64_t kn_t, kn_h, vn_t, vn_h;
  int64_t k_page, k_key, k_head, v_page, v_key, v_head;
};

// Rows to or from pools in four bits (page_mxfp4.hip): strides in elements, those of the scales are the pools' / 32.
struct PageMxfp4Args {
  void* k_rows; void* v_rows; const int64_t* slots;
  uint8_t* k_pages; uint8_t* v_pages; uint8_t* k_block; uint8_t* v_block;
  int heads, page_shift;
  int64_t n_slots, tokens;
  int64_t kn_t, kn_h, vn_t, vn_h;
  int64_t k_page, k_key, k_head, v_page, v_key, v_head;
};

// Paged attention.  The rows of a request (its new tokens times the query heads of a KV head) are taken
// in row tiles of whole tokens (tile_tokens each; where one token has more heads than a tile has rows,
// head_blocks tiles per token).  An item is a row tile of one request and KV head; its keys are counted
// in tiles.  Lengths are known on the device alone, so every workgroup works out by itself what it takes; a request is
// charged its keys as if all its row tiles reached the last one.
// Few rows: the items of a KV head, one behind the other, are cut into equal shares; a workgroup takes a share, whole
// items and parts of the first and the last, of a set of one, two, four or eight KV heads at once, by different ones of its eight
// wavefronts.  A partial of either goes to the workspace (slots 2 i and 2 i + 1 of share and KV head i), and the
// workgroup that finds all others of the item there joins them.
// Many rows: a long item is cut into pieces, one workgroup each, joined by a second kernel.  Pieces get 1/target of the sum or
// somewhat more, so that there are no more than `target` of them where the items allow it; a request that is cut has more than
// piece_tiles tiles per item, so cut items have at most twice target pieces together.
struct PagedArgs {
  const void* q; const void* k; const void* v; const float* k_scale; const float* v_scale;
  const int* table; const int* lengths; const int* token_start;
  void* out; float* lse; float* partial;
  int batch, Hq, Hkv, G, page_shift, max_pages, max_new, n_sink, n_local;
  int max_len, max_tokens, n_pages;
  int tile_tokens, head_blocks;
  float scale_log2;       // logits scale * log2(e)
  float per_piece;        // (1 + margin) / target pieces
  int target;             // pieces, or shares of all sets
  int min_tiles;          // key tiles of one at least
  int slots;              // partials that there is room for
  int near_shift, set_shift, group_shift, shares[kPagedGroupShift + 1];   // few rows: see PagedForm
  unsigned* arrived;      // few rows: partials of the cut item that begins in a share which are there (0 between calls)
  int64_t k_page, k_key, k_head, v_page, v_key, v_head, q_t, q_h;
  // Pools in four bits: scales, whose strides are those of the elements / 32; strides in rows of 128 elements; whether both pools have the same.
  const uint8_t* k_block; const uint8_t* v_block;
  uint32_t k_page_rows, k_key_rows, v_page_rows, v_key_rows;
  int same_strides;
};

// Accounts of attention weight (page_weights.hip).
struct PageWeightsArgs {
  PagedArgs paged;
  const float* lse; const int* counted; float* weights;
  int heads;              // KV heads that a workgroup takes at once; many rows: shares of the rows
};

// Which keys stay (page_keep.hip).
struct PageKeepArgs {
  const float* weights; const int* table; const int* lengths; const int* budgets;
  int* kept; int* lengths_out;
  int batch, heads, page_shift, max_pages, max_len, n_pages, n_first, n_last, max_keep;
  int parts;              // workgroups to a request's KV head
  void* workspace;        // of several: what they tell one another
};

// Eviction (page_evict.hip).  An array of rows in the pages: strides in bytes; a row is `slices` slices of `slice` bytes.
struct PagedArray {
  char* at;
  int64_t page, key, head;
  int slice, slices;
};
constexpr int kEvictArrays = 5;
struct PageEvictArgs {
  const int* kept; const int* lengths; const int* stay; const int* table; int* free_pages; const int* n_free;
  int* n_free_out; int* status;
  int batch, heads, page_shift, max_pages, max_len, max_keep;
  int64_t n_pages;
  PagedArray arrays[kEvictArrays];
};

struct PagedRequest {
  int len, tokens, row;   // keys, new tokens, row of the first one
};

__device__ inline PagedRequest paged_request(const PagedArgs& a, int b) {
  PagedRequest r;
  const int len = a.lengths[b];
  r.len = len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
  if (a.token_start) {
    const int s0 = a.token_start[b], s1 = a.token_start[b + 1];
    r.row = s0 < 0 ? 0 : (s0 > a.max_tokens ? a.max_tokens : s0);
    const int end = s1 < r.row ? r.row : (s1 > a.max_tokens ? a.max_tokens : s1);
    r.tokens = end - r.row < a.max_new ? end - r.row : a.max_new;
  } else {
    r.row = b;
    r.tokens = 1;
  }
  return r;
}

__device__ inline int paged_row_tiles(const PagedArgs& a, int tokens) {
  return (tokens + a.tile_tokens - 1) / a.tile_tokens * a.head_blocks;
}

// Key tiles that a row tile of the request has at most (what its items are charged).
template <int KT>
__device__ inline int paged_charge(const PagedArgs& a, int len) {
  int n = (len + KT - 1) / KT;
  if (a.n_local > 0) {
    const int w = (a.n_sink + KT - 1) / KT + (a.n_local + a.tile_tokens - 2) / KT + 2;
    n = n < w ? n : w;
  }
  return n > 1 ? n : 1;
}

// The key tiles of one row tile, tokens first .. last of the request: the sink's, then those of the window.
// Tile v of `count` is tile v of the cache, or v + skip from `sink` on.
struct PagedSpan {
  int count, sink, skip;
};
template <int KT>
__device__ inline PagedSpan paged_span(const PagedArgs& a, int len, int tokens, int first, int last) {
  PagedSpan s{0, 0, 0};
  const int end = len - tokens + last + 1;               // one behind the last key attended
  if (end <= 0) return s;
  s.count = (end + KT - 1) / KT;
  if (a.n_local > 0) {
    const int lo = len - tokens + first - a.n_local + 1;
    if (lo > 0) {
      const int kept = a.n_sink < lo ? a.n_sink : lo, sink = (kept + KT - 1) / KT, from = lo / KT;
      if (from > sink) {
        s.sink = sink;
        s.skip = from - sink;
        s.count -= s.skip;
      }
    }
  }
  return s;
}

struct PagedPiece {
  int b, g, tile, piece, pieces;   // request, KV head, row tile, piece of the item and how many it has
  PagedRequest r;
  int slot;                        // of the item's first partial
};

// Inclusive prefix sums over the wavefront's lanes.
__device__ inline int wave_prefix(int v) {
  v = half_prefix_sum32(v);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
}

// Many rows: which workgroup takes what.  kPieces: all pieces, a KV head's on one XCD (workgroups go to the eight XCDs in turn; where
// the number of KV heads goes with eight), whose L2 then serves the row tiles that read the same keys.  kCutItems: the items
// that are cut, for the join.
enum { kPieces, kCutItems };

// What workgroup `index` takes; called by whole wavefronts, false where there is nothing.
template <int KT, int WHAT>
__device__ inline bool paged_locate(const PagedArgs& a, int index, PagedPiece& out) {
  const int lane = threadIdx.x & 63;
  out.g = index % a.Hkv;
  index /= a.Hkv;
  float total = 0.f;
  int longest = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    float cost = 0.f;
    if (b < a.batch) {
      const PagedRequest r = paged_request(a, b);
      const int charge = paged_charge<KT>(a, r.len);
      cost = (float)paged_row_tiles(a, r.tokens) * (float)a.Hkv * (float)charge;
      longest = max(longest, charge);
    }
    total += wave_sum(cost);
  }
  const float want = fminf(ceilf(total * a.per_piece), 1073741824.f);
  int piece_tiles = max((int)want, a.min_tiles);
  const bool cut = __any(longest > piece_tiles);
  if (cut && piece_tiles > a.min_tiles) {
    // The smallest of eight lengths that makes no more than target pieces (counted in float32: about), or the first.  Prompt chunks of 128
    // tokens behind 20000, three requests of 32 heads over 8 (96 row tiles): 256 us with the first always, 209; of 64, seven requests at 30000 470 | 376.
    // It costs a workgroup 2 us: two of 512 tokens behind 20000 478 | 478.
    float count[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const float by = __builtin_amdgcn_rcpf((float)piece_tiles);
    for (int b = lane; b < a.batch; b += 64) {
      const PagedRequest r = paged_request(a, b);
      const float tiles = (float)paged_row_tiles(a, r.tokens) * (float)a.Hkv, charge = (float)paged_charge<KT>(a, r.len) * by;
#pragma unroll
      for (int k = 0; k < 8; ++k) count[k] += tiles * ceilf(charge * (8.f / (8 + k)));
    }
    int fits = 0;
#pragma unroll
    for (int k = 7; k >= 0; --k)
      if (wave_sum(count[k]) <= (float)a.target) fits = k;
    piece_tiles += (piece_tiles * (int64_t)fits + 7) / 8;
  }
  if (WHAT == kPieces && cut && a.batch <= 64) {
    // Items with most keys first, over all requests: what is dealt out last is short.  Where items are cut there are few rounds, and the last one
    // shows: 20 ragged chunks of 100 tokens behind up to 60000 962 us in the requests' order, 750 so; ten of 300 behind 30000 766 | 674.
    // Where none is, the order by requests keeps what reads the same keys together: 60 prompts of up to 4096 tokens 1300 | 1342, 16 of up to 8192 1745 | 1754.  An item's level is its tiles up to its last token's key
    // (at most what the request is charged); at_least(x): a request's row tiles of level x or more, the last ones.  The level of the
    // item sought is found by halving.
    PagedRequest r{0, 0, 0};
    int tiles = 0, pieces = 1, top = -1;
    if (lane < a.batch) {
      r = paged_request(a, lane);
      tiles = paged_row_tiles(a, r.tokens);
      const int charge = paged_charge<KT>(a, r.len);
      pieces = (charge + piece_tiles - 1) / piece_tiles;
      top = tiles ? min((r.len + KT - 1) / KT, charge) : -1;
    }
    auto at_least = [&](int x) {
      if (x > top) return 0;
      if (x == 0) return tiles;                            // (more tokens than keys: the first ones attend nothing)
      const int ahead = KT * (x - 1) - (r.len - r.tokens), t = ahead > 0 ? ahead / a.tile_tokens * a.head_blocks : 0;
      return tiles - min(t, tiles - 1);
    };
    auto before = [&](int x) { return __builtin_amdgcn_readlane(wave_prefix(pieces * at_least(x)), 63); };
    if (before(0) <= index) return false;
    int lo = 0, hi = (int)wave_max((float)top) + 1;        // pieces of level lo or more: more than index; of hi or more: not
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before(mid) > index) lo = mid;
      else hi = mid;
    }
    const int many = at_least(lo), more = lo < top ? at_least(lo + 1) : 0, count = pieces * (many - more);
    const int rank = index - before(lo + 1), upto = wave_prefix(count), partials = pieces > 1 ? tiles * pieces : 0, slots = wave_prefix(partials);
    const int f = __ffsll((unsigned long long)__ballot(upto > rank)) - 1;
    auto at = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
    const int i = rank - at(upto - count), here = at(many - more);
    out.b = f;
    out.r.len = at(r.len); out.r.tokens = at(r.tokens); out.r.row = at(r.row);
    out.pieces = at(pieces);
    out.piece = i / here;
    out.tile = at(tiles - many) + i % here;
    out.slot = (at(slots - partials) + out.tile * out.pieces) * a.Hkv + out.g * out.pieces;
    return true;
  }
  int base = 0, slot_base = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    PagedRequest r{0, 0, 0};
    int tiles = 0, pieces = 1;
    if (b < a.batch) {
      r = paged_request(a, b);
      tiles = paged_row_tiles(a, r.tokens);
      pieces = (paged_charge<KT>(a, r.len) + piece_tiles - 1) / piece_tiles;
    }
    const int cut = pieces > 1 ? tiles * pieces : 0;
    const int count = WHAT == kCutItems ? (pieces > 1 ? tiles : 0) : tiles * pieces;
    const int upto = wave_prefix(count), slots = wave_prefix(cut);
    const uint64_t found = __ballot(base + upto > index);
    if (found) {
      const int f = __ffsll((unsigned long long)found) - 1;
      auto at = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
      const int i = index - base - at(upto - count), row_tiles = at(tiles);
      out.b = b0 + f;
      out.r.len = at(r.len); out.r.tokens = at(r.tokens); out.r.row = at(r.row);
      out.pieces = at(pieces);
      out.piece = WHAT == kCutItems ? 0 : i / row_tiles;
      out.tile = row_tiles - 1 - i % row_tiles;          // (the last row tile has most keys: first)
      out.slot = (slot_base + at(slots - cut) + out.tile * out.pieces) * a.Hkv + out.g * out.pieces;
      return true;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
    slot_base += __builtin_amdgcn_readlane(slots, 63);
  }
  return false;
}

// Tiles [begin, end) of an item's `count` that piece `piece` of `pieces` takes.
__device__ inline void paged_piece_range(int count, int piece, int pieces, int& begin, int& end) {
  const int each = count / pieces, more = count % pieces;
  begin = piece * each + (piece < more ? piece : more);
  end = begin + each + (piece < more ? 1 : 0);
}

// Few rows: a workgroup's share of the items of a set of 1 << shift KV heads, in groups of key tiles: [begin, end) of all, which starts
// inside request b, whose items begin at `base`; pos: where the workgroup is.
struct PagedShare {
  int set, shift, j, b, base, pos, begin, end, each;
  PagedRequest r;
};
// The item that `pos` lies in: its first group, and the groups [from, to) of its `groups` that the share has.
struct PagedItem {
  int set, shift, group_shift, b, tile, begin, from, to, groups;
  PagedRequest r;
};

// (the host chooses group_shift so that the groups of all row tiles stay below 2^31)
template <int KT>
__device__ inline int paged_groups(const PagedArgs& a, int len, int group_shift) {
  return (paged_charge<KT>(a, len) + (1 << group_shift) - 1) >> group_shift;
}

// How many KV heads a workgroup takes at once, by different wavefronts, follows from the parts that the longest item is cut into: a set's parts are
// joined by one workgroup.  Measured, us, a head at a time | in sets, 4 query heads a KV head if not said otherwise:
//   Where a token's rows of several heads lie one behind the other, wavefronts that read them at about the same time read longer runs of memory
//   (e4m3 rows of 128 bytes, eight heads, plain reads: 5.5 TB/s by one head, 6.3 by two, 6.7 by four, whether a wavefront takes all of them or each its
//   own).  So up to 512 bytes, at up to 16 parts, if there are 16 key tiles or more for each wavefront: e4m3, 8 KV heads, 48 requests of up to 30011
//   keys and 8 query heads 111 | 103, 16 x 8192 60.5 | 55.7; 32 KV heads, 4 x 20000 136 | 117, 64 x 2000 220 | 168; bf16, 64 x 4000 179 | 170.  At 32
//   parts and more the join costs more: 1 x 65536 38 | 42 in twos, 68 in fours; at four tiles a wavefront it does too: 32 KV heads, 1 x 8192 22.5 | 24.3.
//   Query rows of a set beyond the 32 that are joined at once: 16 x 4096, 32 rows 39.9 | 69.
//   Where items are short, at most a share, sets of any heads save the way from item to item: 8 KV heads, 256 x 300 e4m3 62 | 36, bf16 77 | 58, stored
//   head by head 59 | 35, 1000 x 50 171 | 52, 32 rows 256 x 300 84 | 51.
//   Four bits: two heads' rows share a line of 128 bytes and eight heads' scales do, so sets pay from two tiles for each wavefront on (and lines are kept in
//   the caches): 8 KV heads, token by token, 48 requests of up to 30011 keys 106 | 88, 16 x 16384 89 | 79.
// The sets of a share follow one another on one XCD (workgroups go to the eight XCDs in turn).
// SETS: whether it may be more than one (the way there costs a small call 0.5 us, of 12).
template <int KT, bool SETS>
__device__ inline bool paged_share(const PagedArgs& a, int index, PagedShare& out) {
  const int lane = threadIdx.x & 63;
  PagedRequest r0{0, 0, 0};                                 // (the first 64 requests are read once)
  if (lane < a.batch) r0 = paged_request(a, lane);
  int shift = 0, shares = a.shares[0];
  if constexpr (SETS) {
    float sum = 0.f, longest = 0.f;
    for (int b = lane; b < a.batch; b += 64) {
      const PagedRequest r = b < 64 ? r0 : paged_request(a, b);
      const float charge = r.tokens > 0 ? (float)paged_charge<KT>(a, r.len) : 0.f;
      sum += charge * (float)paged_row_tiles(a, r.tokens);
      longest = fmaxf(longest, charge);
    }
    sum = wave_sum(sum) * (float)a.Hkv;
    longest = wave_max(longest) * (float)a.target;
    const float near = sum * (sum >= (float)(paged_near_tiles(KT) * a.target) ? (float)kPagedNearParts : 1.f);
    while (shift < a.set_shift && longest * (float)(2 << shift) <= (shift < a.near_shift ? near : sum)) ++shift;
    shift = __builtin_amdgcn_readfirstlane(shift);
#pragma unroll
    for (int x = 1; x <= kPagedGroupShift; ++x) shares = shift == x ? a.shares[x] : shares;
  }
  out.shift = shift;
  const int group_shift = a.group_shift - shift;
  const int sets = a.Hkv >> shift, i = index >> 3;
  out.set = i % sets;
  out.j = i / sets * 8 + (index & 7);
  if (out.j >= shares) return false;
  auto groups_of = [&](const PagedRequest& r) { return paged_row_tiles(a, r.tokens) * paged_groups<KT>(a, r.len, group_shift); };
  int total = 0;
  for (int b0 = 64; b0 < a.batch; b0 += 64) {             // (the first 64 requests are counted below, once)
    const int b = b0 + lane;
    total += __builtin_amdgcn_readlane(wave_prefix(b < a.batch ? groups_of(paged_request(a, b)) : 0), 63);
  }
  int base = 0;
  out.each = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    PagedRequest r = r0;
    if (b0 > 0) {
      r = PagedRequest{0, 0, 0};
      if (b < a.batch) r = paged_request(a, b);
    }
    const int v = groups_of(r), upto = wave_prefix(v), all = __builtin_amdgcn_readlane(upto, 63);
    if (b0 == 0) {
      total += all;
      if (total == 0) return false;
      out.each = (int)(((uint32_t)total + (uint32_t)shares - 1u) / (uint32_t)shares);
      const int64_t begin = (int64_t)out.each * out.j;
      if (begin >= total) return false;
      out.begin = out.pos = (int)begin;
      out.end = out.each < total - out.begin ? out.begin + out.each : total;
    }
    const uint64_t found = __ballot(base + upto > out.begin);
    if (found) {
      const int f = __ffsll((unsigned long long)found) - 1;
      out.b = b0 + f;
      out.r.len = __builtin_amdgcn_readlane(r.len, f);
      out.r.tokens = __builtin_amdgcn_readlane(r.tokens, f);
      out.r.row = __builtin_amdgcn_readlane(r.row, f);
      out.base = base + __builtin_amdgcn_readlane(upto - v, f);
      return true;
    }
    base += all;
  }
  return false;
}

// (the share lies in LDS: the same for all lanes)
__device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <int KT, bool SETS>
__device__ inline PagedItem paged_item(const PagedArgs& a, const PagedShare& s) {
  PagedItem i;
  i.set = uniform(s.set);
  i.shift = SETS ? uniform(s.shift) : 0;
  i.group_shift = a.group_shift - i.shift;
  i.b = uniform(s.b);
  i.r.len = uniform(s.r.len); i.r.tokens = uniform(s.r.tokens); i.r.row = uniform(s.r.row);
  const int tiles = paged_row_tiles(a, i.r.tokens), pos = uniform(s.pos), base = uniform(s.base), end = uniform(s.end);
  i.groups = paged_groups<KT>(a, i.r.len, i.group_shift);
  const int k = tiles > 1 ? (pos - base) / i.groups : 0;
  i.begin = base + k * i.groups;
  i.from = pos - i.begin;
  i.to = min(i.groups, end - i.begin);
  i.tile = k & 1 ? tiles - 1 - k / 2 : k / 2;              // (from both ends in turn: later tokens have more keys)
  return i;
}
// Behind the item, by one whole wavefront: the next request that has rows, if the share goes on there (requests without rows, idle places of a
// batch, are passed by 64 at a time).
template <int KT, bool SETS>
__device__ inline void paged_next(const PagedArgs& a, PagedShare& s) {
  const int lane = threadIdx.x & 63;
  bool idle = false;
  if (lane == 0) {
    const int tiles = paged_row_tiles(a, s.r.tokens), groups = paged_groups<KT>(a, s.r.len, a.group_shift - (SETS ? s.shift : 0));
    const int next = s.base + tiles * groups, k = tiles > 1 ? (s.pos - s.base) / groups : 0;
    s.pos = min(s.base + (k + 1) * groups, s.end);
    if (s.pos < s.end && s.pos == next) {
      s.base = next;
      if (++s.b < a.batch) {
        s.r = paged_request(a, s.b);
        idle = s.r.tokens == 0;
      } else {
        s.pos = s.end;                                     // (not reached while the requests stay as they were counted)
      }
    }
  }
  if (!__any(idle)) return;
  for (int b0 = uniform(s.b) + 1; b0 < a.batch; b0 += 64) {
    PagedRequest x{0, 0, 0};
    if (b0 + lane < a.batch) x = paged_request(a, b0 + lane);
    const uint64_t found = __ballot(x.tokens > 0);
    if (!found) continue;
    if (lane == __ffsll((unsigned long long)found) - 1) { s.b = b0 + lane; s.r = x; }
    return;
  }
  if (lane == 0) s.pos = s.end;
}

// A partial's maximum as it is stored: an empty partial has -inf, and the join leaves it out.  One whose scores are all NaN has found no
// maximum either, but its sum is NaN.
__device__ inline float paged_partial_max(float m, float l) { return m == -INFINITY && l != 0.f ? 0.f : m; }

// Eight elements, e0 .. e0 + 7, of a finished row: o / l (times the values' scale), and with the first ones the row's lse.  A row that no key has
// a weight in is zeros, whatever is in o: logits of -inf at keys whose values are infinite leave a NaN there.
template <bool FP32>
__device__ inline void paged_write_row(const PagedArgs& a, int64_t row, int e0, const float (&o)[8], float m, float l, float v_scale) {
  const bool none = l == 0.f;                              // (a NaN is not)
  const float by = v_scale / l;
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = none ? 0.f : o[e] * by;
  if constexpr (FP32) {
    float4* to = reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + row * kHeadDim + e0);
    to[0] = make_float4(x[0], x[1], x[2], x[3]);
    to[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
    *reinterpret_cast<bf16x8*>(reinterpret_cast<uint16_t*>(a.out) + row * kHeadDim + e0) = v;
  }
  if (a.lse && e0 == 0) a.lse[row] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t s);
hipError_t launch_page_append(const PageAppendArgs& a, hipStream_t s);
hipError_t launch_page_append_mxfp4(const PageMxfp4Args& a, hipStream_t s);
hipError_t launch_page_read_mxfp4(const PageMxfp4Args& a, hipStream_t s);
hipError_t launch_page_weights(const PageWeightsArgs& a, int element, const WeightsForm& form, hipStream_t s);
hipError_t launch_page_keep(const PageKeepArgs& a, int64_t rows, hipStream_t s);
hipError_t launch_page_evict(const PageEvictArgs& a, hipStream_t s);
void launch_paged_many_rows(const PagedArgs& a, int element, const PagedForm& form, hipStream_t s);
hipError_t launch_paged_attention(const PagedArgs& a, int element, const PagedForm& form, hipStream_t s);

}  // namespace mp
