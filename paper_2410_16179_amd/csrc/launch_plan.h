// Rules by which the launchers choose a form from the sizes alone, host code without the HIP runtime.
#pragma once
#include <cstddef>
#include <cstdint>

namespace mp {

constexpr int kNumCU = 256;           // MI355X
constexpr int kRangeBlocks = 16;      // key blocks whose ballots a gather wavefront expands at a time (1024 keys)

// The separate gather of the table form: every head is taken by `runs` wavefronts of `run_blocks` key blocks each, and
// its static keys are dealt over them (static_runs = 0), or over static_runs wavefronts of their own, static_keys
// neighbouring ones each.  full: the form that takes full batches of rows through code of their own.
struct GatherPlan { int run_blocks, runs, static_runs, static_keys; bool full; };

// Key blocks of a gather wavefront, in pieces of kRangeBlocks.  A wavefront that takes several pieces fills its
// batches of rows (a piece samples about 20 keys of a batch's 32 at 2 %), asks for the next piece's ballots early
// and leaves one partial: as many pieces as bring all wavefronts into one round, sixteen per compute unit.
// Measured (us per step through tables, pieces 1 | 2 | 3 | 4 | 8): 512 heads x 131072 keys, (10,170), - | 181 | - | 166.5 |
// 161.8 (16: 162.5); (10,150): 512 x 32768 62.9 | 59.6 | 59.3 | 58.2 | 58.0; 128 x 65536
// 43.6 | 42.4 | 42.5 | 43.1 | 47.4; 64 x 98304 42.4 | 40.6 | 39.2 | 40.6 | 48.6; 256 x 20000, (9,120), 46.0 | 45.6 | 45.5 | 49.5 |
// 60.8; 512 x 30000, (9,100), six pieces (five runs, 1.25 workgroups per compute unit) 86.6, four 78.0.
constexpr int64_t kGatherWaves = 16 * kNumCU;
constexpr int64_t kMaxGatherPieces = 8;
// Static keys.  Up to 16 of them, half a batch, join a run's last batch.  More cost it batches of their own, one after
// the other, so they go to wavefronts of their own while the chip has room: of 32 keys, and of 64 where that leaves the
// fullest SIMD fewer wavefronts, from four on.  Measured, us per step through tables, static keys dealt over the runs |
// own wavefronts of 32 | of 64 (all of 32 contiguous keys and no full batches: the form before runs had several pieces):
// (10,150), 512 heads, 1024 keys, 68 static 25.2 | 18.8 | 19.5 (18.7), 1004 static 119 | 42.3 | 40.0 (41.8); 2048, 68 22.8 |
// 21.4 | 19.9 (20.9); 16384, 4100 147 | 133 | 113 (129); 32 heads, three hits, 16384 keys, 4100 38.2 | 22.7 | 21.5 (22.6), 528
// 18.8 | 16.8 | 17.3 (16.1); 68 16.0 | 16.4 | 16.7 (15.9).
// Where the runs fill the chip by themselves, static keys dealt over them fill their batches, and wavefronts of
// their own only pay for more than two batches per piece: 512 heads, dealt | own of 64 | of 128: 8192 keys, 516 static 36.2 |
// 37.4 | 41.5; 16384, 2004 84.4 | 73.3 | 77.1; 32768, 1092 73.3 | 73.2 | 69.8; 65536, 1004 97.5 | 105.3 | 97.6; 2504
// 141 | 147 | 135; 6004 259 | 198 | 205; (8,75), float32, 32768, 1504 280 | 455 | 313; (9,120), e4m3, 65536, 2504 126 | 161 | 138.
// Full batches through code of their own cost a wavefront that has none 0.4 us (32 heads, 16384 keys, three hits 16.5 |
// 16.0): where one piece of a run samples most of a batch at most, the form without is taken, for any threshold above one hit.
inline GatherPlan plan_gather(int units, int G, int64_t nblk, int64_t n_static, int tau) {
  const int64_t heads = (int64_t)units * G;
  int64_t pieces = (heads * ((nblk + kRangeBlocks - 1) / kRangeBlocks) + kGatherWaves - 1) / kGatherWaves;
  pieces = pieces < 1 ? 1 : (pieces > kMaxGatherPieces ? kMaxGatherPieces : pieces);
  GatherPlan p;
  p.run_blocks = (int)pieces * kRangeBlocks;
  p.runs = (int)((nblk + p.run_blocks - 1) / p.run_blocks);
  p.full = pieces > 1 || tau == 1;
  p.static_runs = 0;
  p.static_keys = 32;
  auto wavefronts = [&](int64_t per_head) {                // of the fullest SIMD
    return (units * per_head + kNumCU - 1) / kNumCU * G / 4;
  };
  auto own = [&](int keys) { return (n_static + keys - 1) / keys; };
  const bool filled = pieces > 1 || wavefronts(p.runs) >= 4;
  if (n_static <= p.runs * (filled ? 64 * pieces : 16)) return p;
  if (filled) p.static_keys = pieces > 2 ? 128 : 64;
  else if (wavefronts(p.runs + own(32)) >= 4 && wavefronts(p.runs + own(64)) < wavefronts(p.runs + own(32))) p.static_keys = 64;
  p.full |= p.static_keys > 32;
  p.static_runs = (int)own(p.static_keys);
  return p;
}

// One-launch scan + gather: most workgroups of one head each for which a workgroup serves one of the G > 1 heads of a KV
// head.  Where few workgroups share the chip a wavefront then compares its blocks with one head's code, not with G one after
// the other, and gathers for one head (of five to eight heads a wavefront gathers for two); beyond that reading the
// codes G times costs more.  tuned: table sets with a scan of their own.  us of scan + gather and merge, G heads a
// workgroup | one (workgroups of one head): G = 2, 8 KV heads, (10,150): 4096 keys 10.5 | 9.9 (256), 6144 10.5 | 10.4 (384), 8192 10.5 | 10.9 (512);
// (9,110) 8192 13.5 | 13.5 (512).  G = 3: 4096 10.6 | 10.3 (384), (8,75), float32, 5400 12.8 | 12.0 (528); step, 10000 19.2 | 20.0 (960).
// G = 4: 2048 step 19.0 | 16.7 (256), 6144 11.1 | 11.1 (768), step 10000 19.8 | 21.1 (1280); any K and L: 4096 step 20.8 | 19.5 (512), 6144
// 13.0 | 13.8 (768).  G = 5: 4096 13.9 | 10.8 (640), 6400 13.9 | 12.5 (1000), (10,100) 16.5 | 15.1; G = 6: (9,120) 5400 15.3 | 12.3 (1056);
// G = 7, 4 KV heads: 9000 14.5 | 12.2 (1008); G = 8: 4000 14.9 | 12.1 (1024), (10,100) 16.8 | 15.0, step 8000 25.2 | 26.0 (2048).
inline int64_t head_per_workgroup_limit(bool tuned, int G) {
  if (G > 4) return 4 * kNumCU;
  return (G == 4 && tuned ? 3 : (G == 2 ? 1 : 2)) * kNumCU;
}

// Float32 key hashing: keys of a workgroup, 32 or 64 (in which a projector element serves two matrix instructions), by the
// workgroups of either kind that the fullest compute unit gets: one of 64 keys takes about 1.75 times one of 32.  Below
// five bits per table 32 throughout: a workgroup is K wavefronts, and many small ones hide each other's latencies.
// us of the kernel, workgroups of 32: 32 keys | 64 keys: 257 (4,32) 11.1 | 12.5; 512 (2,32) 11.4 | 13.6; 1000 (2,64) 12.5 | 18.2; 8192 (4,100)
// 114 | 121; 282 (5,75) 15.6 | 16.0, 1002 35.7 | 25.4; 320 (10,150) 24.9 | 20.9, 515 35.1 | 39.2, 770 46.3 | 39.7, 2560 115.9 | 97.5;
// 384 (8,75) 16.9 | 16.5, 768 24.2 | 27.3, 1536 44.5 | 40.1; 640 (9,100) 35.7 | 39.0, 1272 58.8 | 57.6; 258 (16,64) 29.8 | 26.1, 750 46.2 | 50.8.
inline int hash_f32_keys(int K, int64_t groups32, int64_t groups64) {
  auto fullest = [](int64_t groups) { return (groups + kNumCU - 1) / kNumCU; };
  return K >= 5 && 7 * fullest(groups64) < 4 * fullest(groups32) ? 64 : 32;
}

// ---- page plan -----------------------------------------------------------------------------------------
// Workgroups of a step's page plan in one launch, every one with all prefix sums in its LDS; 0: two launches, sums first.  Several
// workgroups need inputs that are not written over.  Measured, us a call in a graph, one launch | two: 64 requests of one token 3.2 | 4.9, 2000 of
// one 6.2 | 13.8, 2000 of up to 100 (eight in ten of one) 8.8 | 16.6, 8 of up to 2048 4.1 | 6.2; 512 of up to 2048 (35840 rows) 5.8 | 9.5, in 8
// workgroups for 35 13.1.  Written in place, one workgroup: 8 x 250 rows 3.9 | 5.4, 8 x 500 5.2 | 5.5, 64 x 64 6.0 | 5.9, 512 x 8 7.1 | 7.3,
// 64 x 125 9.4 | 6.0.
constexpr int kPlanInOneRequests = 2048, kPlanInOneTokens = 4096, kPlanMostWorkgroups = 128;
inline int page_plan_workgroups(int batch, int64_t max_tokens, bool in_place) {
  if (batch > kPlanInOneRequests) return 0;
  if (in_place) return max_tokens <= kPlanInOneTokens ? 1 : 0;
  const int64_t n = (max_tokens + 1023) / 1024;
  return n <= 2 ? 1 : (int)(n < kPlanMostWorkgroups ? n : kPlanMostWorkgroups);
}
// Whether either kind of call may need the workspace.
inline bool page_plan_needs_workspace(int batch, int64_t max_tokens) { return page_plan_workgroups(batch, max_tokens, true) == 0; }

// ---- paged attention ------------------------------------------------------------------------------
constexpr int kPagedGroupShift = 3, kPagedGroup = 1 << kPagedGroupShift;   // few rows: wavefronts of a workgroup
// Few rows: near_shift, set_shift: KV heads that a workgroup may take at once (1 << each), for the two reasons that paged_share knows; group_shift: 1 <<
// that many key tiles are a group, by which work is shared, for one KV head (of sets, as many fewer as heads more); shares: of a set of 1 << index KV heads.
// rows: query rows (new tokens times the query heads of a KV head) that a workgroup takes at once; key_tile:
// keys by which the work is counted.  tile_tokens, head_blocks: see PagedArgs.  target: pieces that the work is cut into;
// min_tiles: key tiles of a piece at least.  items, pieces, units, slots: at most so many row
// tiles of all KV heads, workgroups, row tiles that are cut, partials.
struct PagedForm {
  int rows, key_tile, tile_tokens, head_blocks, target, min_tiles, near_shift, set_shift, group_shift, shares[kPagedGroupShift + 1];
  int64_t items, pieces, units, slots;
};

// Up to 32 rows are taken by the form that keeps keys in registers, 16 or 32 at a time; more (bf16) by the one that shares
// keys among 128 rows through LDS.  float32: always 16, for which prompts pay: every sixteen rows read the keys again (four prompts of up to 4099 tokens 5.4 ms,
// 54 TFLOP/s, 512 tokens behind 8000 708 us, 98 TFLOP/s, of the 153 of a library product).  Measured, us, requests x keys, 32 heads over 8: up to 16 rows taken 16 | 32 at a time: 1 x 2048
// (4 rows) 12.5 | 14.3, 1 x 98304 79.0 | 81.5, 16 x 4096 (16 rows) 54.4 | 56.4; 17 to 32 rows 16 | 32 at a time | by the form for many: 20 rows 16 x 4096 94.7 | 57.2
// | 67.1, 32 rows 1 x 65536 78.2 | 76.9 | 76.6, 64 x 1000 96.6 | 54.0 | 62.7; 36 rows 32 at a time | by the form for many: 16 x 4096 97 | 70.7, 64 x 300
// 37.5 | 24.4, 1 x 65536 85.5 | 80.9, 1 x 2048 19.8 | 24.5; 64 rows 64 x 1000 91.5 | 66.5, 1 x 65536 86.9 | 92.1.
constexpr int kPagedManyRows = 128, kPagedManyKeys = 64;
constexpr int kPagedNearParts = 16, kPagedNearTiles = 128;   // few rows: see paged_share
constexpr int kPagedFourTile = 64;           // few rows, pools in four bits: keys of a tile
constexpr int paged_near_tiles(int tile) { return tile == kPagedFourTile ? 16 : kPagedNearTiles; }
constexpr int kPagedCounters = 1024;         // words at the start of the workspace, one per share (at most kNumCU, or one for each KV head)
inline int paged_rows(bool fp32, int64_t rows) { return fp32 || rows <= 16 ? 16 : (rows <= 32 ? 32 : kPagedManyRows); }

// Row tiles of all KV heads and requests, whatever token counts (each at most max_new) the device memory holds.
inline int64_t paged_most_items(int batch, int kv_heads, int group, bool fp32, int max_new) {
  const int rows = paged_rows(fp32, (int64_t)max_new * group);
  const int64_t tokens = group <= rows ? rows / group : 1, blocks = group <= rows ? 1 : (group + rows - 1) / rows;
  return (int64_t)batch * ((max_new + tokens - 1) / tokens) * blocks * kv_heads;
}

// group: query heads per KV head.  starts: the requests' token counts differ (else one token each).  row_bytes: of a key's row, where the rows of a key's
// heads lie one behind the other in both pools; else 0.
// four: pools in four bits, of which a wavefront takes 64 keys at once.
inline PagedForm paged_form(int batch, int kv_heads, int group, bool fp32, int64_t max_tokens, int max_new, bool starts, int64_t max_len,
                            int n_sink, int n_local, int row_bytes, bool four = false) {
  PagedForm f{};
  f.rows = paged_rows(fp32, (int64_t)max_new * group);
  const bool many = f.rows == kPagedManyRows;
  f.key_tile = many ? kPagedManyKeys : (fp32 ? 16 : (four ? kPagedFourTile : 32));
  f.tile_tokens = group <= f.rows ? f.rows / group : 1;
  f.head_blocks = group <= f.rows ? 1 : (group + f.rows - 1) / f.rows;
  // target: workgroups that are resident at once.  Many rows, us with half as many | these | twice as many, 32 heads over 8: 64 rows over 65536 keys
  // 102 | 94 | 128, 256 over 8192 40.3 | 38.5 | 39.0, 2048 tokens behind 59392 2706 | 2708 | 2725.  Pieces of at least 256 | 512 | 1024 keys: 256 rows
  // over 8192 43.9 | 38.5 | 43.7, 30 x 300 tokens behind 300 162 | 160 | 157.
  f.target = many ? 2 * kNumCU : kNumCU;
  f.min_tiles = 512 / f.key_tile;
  int64_t tiles = (int64_t)batch * ((max_new + f.tile_tokens - 1) / f.tile_tokens);
  if (starts && max_tokens / f.tile_tokens + batch < tiles) tiles = max_tokens / f.tile_tokens + batch;
  f.items = tiles * f.head_blocks * kv_heads;
  int64_t charge = (max_len + f.key_tile - 1) / f.key_tile;
  if (n_local > 0) {
    const int64_t w = (n_sink + f.key_tile - 1) / f.key_tile + (n_local + f.tile_tokens - 2) / f.key_tile + 2;
    charge = charge < w ? charge : w;
  }
  const int64_t most = (charge + f.min_tiles - 1) / f.min_tiles;
  f.pieces = f.items;
  if (most > 1) {
    const int64_t cut = 2 * f.target + 64;
    f.pieces = f.items * most < f.items + cut ? f.items * most : f.items + cut;
    f.slots = f.items * most < cut ? f.items * most : cut;
    f.units = f.items < f.target ? f.items : f.target;
  }
  if (!many) {
    // near_shift: sets of neighbouring rows, 512 bytes at most, of no more query rows than are joined at once; set_shift: sets that the kernel may
    // choose, whatever the lengths
    const int tokens = max_new < f.tile_tokens ? max_new : f.tile_tokens, used = group < f.rows ? group * tokens : f.rows;
    while (row_bytes > 0 && row_bytes << f.near_shift < 512 && used << (f.near_shift + 1) <= 32) ++f.near_shift;
    while (f.set_shift < kPagedGroupShift && kv_heads % (2 << f.set_shift) == 0 &&
           f.target * (2 << f.set_shift) <= f.items * (f.set_shift < f.near_shift && f.items * charge >= paged_near_tiles(f.key_tile) * f.target ? kPagedNearParts : 1))
      ++f.set_shift;
    // (a group has a key tile for each wavefront of a head; the groups of all row tiles are counted in 31 bits, in sets too)
    auto groups = [&](int shift) { return (charge + (1 << shift) - 1) >> shift; };
    f.group_shift = kPagedGroupShift;
    const int64_t row_tiles = (int64_t)batch * ((max_new + f.tile_tokens - 1) / f.tile_tokens) * f.head_blocks;
    while (row_tiles * groups(f.group_shift - f.set_shift) > INT32_MAX - kPagedCounters) ++f.group_shift;
    f.pieces = f.slots = f.units = 0;
    for (int shift = 0; shift <= f.set_shift; ++shift) {
      const int sets = kv_heads >> shift;
      const int64_t least = groups(f.group_shift - shift) * (f.items / kv_heads), most = f.target > sets ? f.target / sets : 1;
      const int64_t shares = most < least ? most : (least > 1 ? least : 1);
      const int64_t pieces = (shares + 7) / 8 * 8 * sets, slots = 2 * shares * kv_heads;   // (dealt to the eight XCDs in rounds of eight)
      f.shares[shift] = (int)shares;
      f.pieces = pieces > f.pieces ? pieces : f.pieces;
      f.slots = slots > f.slots ? slots : f.slots;
    }
  }
  return f;
}

// ---- which keys stay --------------------------------------------------------------------------------
// Measured, us, 64 requests of up to 9001 keys, 256 | 512 | 1024 threads: 26.2 | 19.4 | 25.9.
constexpr int kKeepShort = 16384;            // requests of up to so many keys are gone over by 512 threads, others by 1024
// Workgroups to a KV head: one, or where few heads leave compute units idle one for each 8192 keys that a request may have, up to 16.
constexpr int kKeepMostParts = 16;
constexpr int kKeepPartList = 2048;          // ranks that one lists
constexpr size_t kKeepPartBytes = 2 * 2048 + 4 * kKeepPartList + 16;
inline int keep_parts(int64_t rows, int64_t max_len) {
  const int64_t parts = (max_len + 8191) / 8192;
  if (parts < 4 || rows > 32 || max_len > kKeepMostParts * 65280) return 1;   // (a part's counts have 16 bits)
  return (int)(parts < kKeepMostParts ? parts : kKeepMostParts);
}

// ---- eviction ---------------------------------------------------------------------------------------
// Bytes of a row that a workgroup moves: whole rows, or pieces of 32 bytes at least where requests times KV heads would leave compute units idle.
// Measured, us, 32768 keys to 8192, bf16, eight heads, slices of 32 | 64 bytes: one request 30.4 | 32.8 (both on one card; slices of 32 take 32 to 33 on others), four (which take 64) 79; with a unit's slices on
// different XCDs, slices of 64 | 128 | 256: one request 35.5 | 56 | 103, four 102 | 100 | 163.
inline int evict_slice(int row, int64_t units) {
  int slice = row;
  while (slice > 32 && 2 * units * (row / slice) < kNumCU) slice /= 2;
  return slice;
}

// ---- accounts of attention weight -------------------------------------------------------------------
// rows: query rows of a KV head (new tokens times query heads) that a wavefront has at once: up to 128 (float32: 16), in registers, its keys going by; many: more of
// them, 32 of which go by at a time, the keys in registers.  heads: KV heads that a workgroup's wavefronts take at once; many: shares that they split the rows
// into; tiles: of keys, at most, all KV heads together; workgroups: what is resident at once; many: at most.
constexpr int kWeightsManyWaves = 4;         // wavefronts of a workgroup, many rows
// Rows from which on they split them; where there are few tiles they do so sooner.  Measured, us, 16 requests of 32768 keys, 32 heads over 8, split from 128 rows on | from
// 512 | 1024 | 4096: 160 rows 968 | 425 | 425 | 426, 512 rows 1353 | 1043 | 878 | 878, 1024 rows 1995 | 1984 | 1686 | 1536, 2048 rows - | 3307 | 3306 | 2844; one request of 4096
// keys, 256 rows: split 12.3, not 19.2.
constexpr int kWeightsShareRows = 4096;
constexpr int weights_tile(bool fp32, int bits, int rows) { return fp32 ? 16 : (bits == 16 || rows > 16 ? 32 : 64); }   // keys of a tile, few rows
struct WeightsForm {
  bool many;
  int rows, heads;
  int64_t tiles, workgroups;
};
inline WeightsForm weights_form(int batch, int kv_heads, int group, bool fp32, int bits, int max_new, int64_t max_len) {
  WeightsForm f{};
  const int64_t rows = (int64_t)max_new * group;
  f.many = rows > (fp32 ? 16 : 128);
  f.rows = 16;
  while (f.rows < 128 && f.rows < rows) f.rows *= 2;
  f.heads = 1;
  int tile = weights_tile(fp32, bits, f.rows);
  int64_t most = (f.rows <= 32 ? 2 : 1) * kNumCU;
  if (f.many) {
    // a workgroup's wavefronts split the rows of one tile of keys, or have tiles of their own
    const int own = fp32 ? 32 : 64;
    auto blocks = [&](int shares) { return (max_len + own * (kWeightsManyWaves / shares) - 1) / (own * (kWeightsManyWaves / shares)) * batch * kv_heads; };
    while (f.heads < kWeightsManyWaves && 64 * f.heads <= rows && (kWeightsShareRows * f.heads <= rows || blocks(f.heads) < 2 * kNumCU)) f.heads *= 2;
    tile = own * (kWeightsManyWaves / f.heads);
    most = 1 << 14;
  } else {
    while (f.heads < 8 && kv_heads % (2 * f.heads) == 0) f.heads *= 2;
  }
  f.tiles = (max_len + tile - 1) / tile * batch * kv_heads;
  f.workgroups = f.tiles < most ? (f.tiles > 0 ? f.tiles : 1) : most;
  return f;
}
// Many rows go by in steps of dt tokens and dh heads of a KV head's `group`.  The wavefront has a 64-bit pointer to the step's first row, a lane 32 bits from there to its own,
// one of 32 behind it: both go on by the step, and by `wrap` (a token's stride less that of `group` heads) where their head goes past the last one.  So a lane's offset stays
// within a token and 126 heads (one head a token: 31 tokens) of the pointer, below 2^31 bytes with strides of up to 2^22 elements, however far the rows reach.
constexpr bool next_head(int& head, int dh, int group) {   // whether it goes past the last one
  head += dh;
  const bool past = head >= group;
  head -= past ? group : 0;
  return past;
}
constexpr int offset_step(bool past, bool first_past, int wrap) { return (past ? wrap : 0) - (first_past ? wrap : 0); }

// Tiles are counted in 31 bits.
inline bool weights_fit(const WeightsForm& f) { return f.tiles <= INT32_MAX - 1024; }

// Whether the form's workgroups make a grid: its threads are counted in 32 bits (those of few rows are a thousand workgroups or a few).
constexpr int kPagedManyThreads = 256;
inline bool paged_grid_fits(const PagedForm& f) { return f.rows != kPagedManyRows || f.pieces * kPagedManyThreads < (int64_t)1 << 32; }

}  // namespace mp
