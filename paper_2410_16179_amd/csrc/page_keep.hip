// Which keys of a request stay: the first ones, the last ones, and those with the largest accounts.
#include "paged_device.h"

namespace mp {
namespace {

constexpr int kLots = 4;                                 // times four keys of a thread are requested at once: a wavefront takes kLots * 256 in order
constexpr int kWaveKeys = kLots * 256;
constexpr int kCopies = 4, kBins = 2048;                 // counts of a digit, in copies for the lanes
constexpr int kList = 8192;                              // ranks of one first digit that are kept in LDS

// The accounts' order as that of unsigned integers: NaN below all, both zeros alike.
__device__ inline uint32_t rank_of(float w) {
  const uint32_t bits = __float_as_uint(w + 0.f);
  const uint32_t up = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
  return w == w ? up : 0u;
}

// A request's KV head.
struct Row {
  const int* table; const float* weights; int* kept;
  int len, stay, first, last;                            // keys [first, last) are chosen by their accounts, `want` of them
  int want;
};
// A request's keys, and those that stay.
struct Size {
  int len, stay;
};
__device__ inline Size size_of(const PageKeepArgs& a, int b) {
  int len = a.lengths[b];
  len = len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
  const int budget = a.budgets[b], most = budget < a.max_keep ? budget : a.max_keep;
  return Size{len, budget < 0 || len <= most ? len : most};
}
__device__ inline Row row_of(const PageKeepArgs& a, int b, int g) {
  const Size n = size_of(a, b);
  const int len = n.len;
  Row r{a.table + (int64_t)b * a.max_pages, a.weights + ((int64_t)g << a.page_shift), a.kept + ((int64_t)b * a.heads + g) * a.max_keep, len, n.stay, a.n_first,
        len - a.n_last, 0};
  if (r.first >= r.last) r.first = r.last = len;           // (no key is chosen by its account)
  r.want = max(r.stay - (len - (r.last - r.first)), 0);
  return r;
}

// Ranks of the lane's keys base + 256 k + 4 lane + e; 0 from `end` on and on pages that are none.
typedef u32x4 Ranks[kLots];
__device__ inline void load_ranks(const PageKeepArgs& a, const Row& r, int base, int end, Ranks& rank) {
  const int mask = (1 << a.page_shift) - 1, lane = threadIdx.x & 63;
  int id[kLots];
#pragma unroll
  for (int k = 0; k < kLots; ++k) {
    const int i = base + 256 * k + 4 * lane;
    id[k] = i < end ? r.table[i >> a.page_shift] : -1;
  }
  f32x4 w[kLots];
#pragma unroll
  for (int k = 0; k < kLots; ++k) {
    w[k] = f32x4{NAN, NAN, NAN, NAN};
    if ((uint32_t)id[k] < (uint32_t)a.n_pages)
      w[k] = *reinterpret_cast<const f32x4*>(r.weights + (((int64_t)id[k] * a.heads) << a.page_shift) + ((base + 256 * k + 4 * lane) & mask));
  }
#pragma unroll
  for (int k = 0; k < kLots; ++k) rank[k] = u32x4{rank_of(w[k][0]), rank_of(w[k][1]), rank_of(w[k][2]), rank_of(w[k][3])};
}
__device__ inline int my_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// f(rank) for the keys [from, to) that are chosen by their accounts; the first ranks, a thread's in `held`, are there already.
template <int THREADS, class F>
__device__ inline void each_rank(const PageKeepArgs& a, const Row& r, int from, int to, const Ranks& held, F&& f) {
  const int lane = threadIdx.x & 63, lo = max(from, r.first), hi = min(to, r.last);
  auto take = [&](int base, const Ranks& rank) {
    const bool all = base >= lo && base + kWaveKeys <= hi;
#pragma unroll
    for (int k = 0; k < kLots; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = base + 256 * k + 4 * lane + e;
        if (all || (i >= lo && i < hi)) f(rank[k][e]);
      }
  };
  int base = from + kWaveKeys * my_wave();
  take(base, held);
#pragma unroll 1
  for (base += kLots * 4 * THREADS; base < to; base += kLots * 4 * THREADS) {
    Ranks rank;
    load_ranks(a, r, base, to, rank);
    take(base, rank);
  }
}

struct Counts {
  int bins[kBins][kCopies];                              // (a digit's copies in different banks: accounts that are alike wait less for one another)
  uint32_t totals[16];
  int found[3], listed;
};
template <int THREADS>
__device__ inline void clear(Counts& c, int size) {
  for (int i = threadIdx.x; i < size; i += THREADS) *reinterpret_cast<u32x4*>(c.bins[i]) = u32x4{0, 0, 0, 0};
  __syncthreads();
}
__device__ inline void count(Counts& c, uint32_t digit) { atomicAdd(&c.bins[digit][threadIdx.x & (kCopies - 1)], 1); }

// From the largest digit down, the one at which `want` keys are reached: found = the digit, keys above it, keys of it.  own: counts of the thread's digits,
// size - 1 - kEach threadIdx.x - d.
template <int THREADS>
__device__ inline void find_digit(Counts& c, int size, int want, const int (&own)[kBins / THREADS]) {
  constexpr int kEach = kBins / THREADS;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = size - 1 - kEach * (int)threadIdx.x;
  int sum = 0;
#pragma unroll
  for (int d = 0; d < kEach; ++d) sum += own[d];
  const int upto = wave_prefix(sum);
  if (lane == 63) c.totals[wave] = (uint32_t)upto;
  __syncthreads();
  int before = upto - sum;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) before += w < wave ? (int)c.totals[w] : 0;
#pragma unroll
  for (int d = 0; d < kEach; ++d) {
    if (before < want && before + own[d] >= want) {
      c.found[0] = at - d;
      c.found[1] = before;
      c.found[2] = own[d];
    }
    before += own[d];
  }
  __syncthreads();
}
__device__ inline int all_copies(const Counts& c, int digit) {
  const u32x4 x = *reinterpret_cast<const u32x4*>(c.bins[digit]);
  return (int)(x.x + x.y + x.z + x.w);
}
template <int THREADS>
__device__ inline void find_counted(Counts& c, int size, int want) {
  constexpr int kEach = kBins / THREADS;
  const int at = size - 1 - kEach * (int)threadIdx.x;
  int own[kEach];
#pragma unroll
  for (int d = 0; d < kEach; ++d) own[d] = at - d >= 0 ? all_copies(c, at - d) : 0;
  find_digit<THREADS>(c, size, want, own);
}

// The digits of 11 and 10 bits below the first one, from a list of the ranks that share it.
template <int THREADS>
__device__ inline void lower_digits(Counts& c, const uint32_t* list, int n, uint32_t& bar, int& want) {
#pragma unroll 1
  for (int digit = 1; digit < 3; ++digit) {
    const int shift = digit == 1 ? 10 : 0, size = digit == 1 ? kBins : 1024;
    clear<THREADS>(c, size);
    for (int i = threadIdx.x; i < n; i += THREADS)
      if (digit == 1 || list[i] >> 10 == bar >> 10) count(c, list[i] >> shift & (size - 1));
    __syncthreads();
    find_counted<THREADS>(c, size, want);
    bar |= (uint32_t)c.found[0] << shift;
    want -= c.found[1];
    __syncthreads();
  }
}

// The bar, the smallest rank that stays, of a whole request, and how many keys of that rank stay (the first ones): by counting digits of 11, 11 and 10 bits
// from the top; keys that share the bar's first digit are looked at in LDS where there is room for them.
template <int THREADS>
__device__ inline void find_bar(const PageKeepArgs& a, const Row& r, Counts& c, uint32_t* list, const Ranks& held, uint32_t& bar, int& want) {
  clear<THREADS>(c, kBins);
  each_rank<THREADS>(a, r, 0, r.len, held, [&](uint32_t rank) { count(c, rank >> 21); });
  if (threadIdx.x == 0) c.listed = 0;
  __syncthreads();
  find_counted<THREADS>(c, kBins, want);
  bar = (uint32_t)c.found[0] << 21;
  want -= c.found[1];
  const int same = c.found[2];
  __syncthreads();
  if (same <= kList) {
    each_rank<THREADS>(a, r, 0, r.len, held, [&](uint32_t rank) {
      if (rank >> 21 == bar >> 21) list[atomicAdd(&c.listed, 1)] = rank;
    });
    __syncthreads();
    lower_digits<THREADS>(c, list, same, bar, want);
    return;
  }
#pragma unroll 1
  for (int digit = 1; digit < 3; ++digit) {
    const int shift = digit == 1 ? 10 : 0, size = digit == 1 ? kBins : 1024, above = digit == 1 ? 21 : 10;
    clear<THREADS>(c, size);
    each_rank<THREADS>(a, r, 0, r.len, held, [&](uint32_t rank) {
      if (rank >> above == bar >> above) count(c, rank >> shift & (size - 1));
    });
    __syncthreads();
    find_counted<THREADS>(c, size, want);
    bar |= (uint32_t)c.found[0] << shift;
    want -= c.found[1];
    __syncthreads();
  }
}

// Writes keys of [from, to) that stay, in order.  taken, ties: keys before `from` that stay for sure (the first and the last ones, and those above the bar), and
// those at the bar, of which the first `want` stay.  Both are counted in one word, the latter in its upper half.
template <int THREADS>
__device__ inline void write_kept(const PageKeepArgs& a, const Row& r, Counts& c, int from, int to, const Ranks& held, uint32_t bar, int want, int taken, int ties) {
  const int lane = threadIdx.x & 63, wave = my_wave();
  const bool by_account = r.want > 0;
#pragma unroll 1
  for (int i0 = from; i0 < to; i0 += kLots * 4 * THREADS) {
    const int base = i0 + kWaveKeys * wave;
    Ranks rank;
    if (i0 == from) {
#pragma unroll
      for (int k = 0; k < kLots; ++k) rank[k] = held[k];
    } else {
      load_ranks(a, r, base, to, rank);
    }
    uint32_t mine[kLots], upto[kLots], own = 0;            // four keys: bit e of what stays for sure, bit 16 + e of what is at the bar
#pragma unroll
    for (int k = 0; k < kLots; ++k) {
      mine[k] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = base + 256 * k + 4 * lane + e;
        const bool open = i >= r.first && i < r.last;
        const uint32_t what = !open || (by_account && rank[k][e] > bar) ? 1u << e : (by_account && rank[k][e] == bar ? 1u << (16 + e) : 0u);
        mine[k] |= i < to ? what : 0u;
      }
      const uint32_t n = (uint32_t)__popc(mine[k] & 15u) | (uint32_t)__popc(mine[k] >> 16) << 16;
      const uint32_t sum = (uint32_t)wave_prefix((int)n);
      upto[k] = own + sum - n;
      own += (uint32_t)__builtin_amdgcn_readlane((int)sum, 63);
    }
    if (lane == 0) c.totals[wave] = own;
    __syncthreads();
    uint32_t earlier = 0, all = 0;                         // (counts of up to 16384 keys)
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      const uint32_t t = c.totals[w];
      earlier += w < wave ? t : 0u;
      all += t;
    }
#pragma unroll
    for (int k = 0; k < kLots; ++k) {
      if (!mine[k]) continue;
      const uint32_t before = upto[k] + earlier;
      int sure_before = taken + (int)(before & 0xffffu), same_before = ties + (int)(before >> 16);
      const int i = base + 256 * k + 4 * lane;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int sure = mine[k] >> e & 1, same = mine[k] >> (16 + e) & 1, at = sure_before + min(same_before, want);
        if ((sure || (same && same_before < want)) && at < r.stay) r.kept[at] = i + e;
        sure_before += sure;
        same_before += same;
      }
    }
    taken += (int)(all & 0xffffu);
    ties += (int)(all >> 16);
    __syncthreads();
  }
}

template <int THREADS>
__device__ inline void fill_behind(const PageKeepArgs& a, const Row& r) {
  for (int j = (r.stay == r.len ? 0 : r.stay) + (int)threadIdx.x; j < a.max_keep; j += THREADS) r.kept[j] = -1;
}

// A workgroup per request and KV head.  Bound by one compute unit's instructions and its chain of reads, counts and barriers: 64 requests of 500 to 9001 keys, eight
// heads each (7.5 MB), 19.4 us with 512 threads (256: 26.2, 1024: 25.9); one of 98304 keys 65, of which counting 14, listing 15, writing 30.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void page_keep_kernel(const PageKeepArgs a) {
  __shared__ __align__(16) Counts counts;
  __shared__ uint32_t list[kList];
  const int b = blockIdx.x / a.heads, g = blockIdx.x - b * a.heads;
  const Row r = row_of(a, b, g);
  if (a.lengths_out && g == 0 && threadIdx.x == 0) a.lengths_out[b] = r.stay;
  if (r.stay < r.len) {
    Ranks held;
    uint32_t bar = 0;
    load_ranks(a, r, kWaveKeys * my_wave(), r.len, held);
    int want = r.want;
    if (want > 0) find_bar<THREADS>(a, r, counts, list, held, bar, want);
    write_kept<THREADS>(a, r, counts, 0, r.len, held, bar, want, 0, 0);
  }
  fill_behind<THREADS>(a, r);
}

// ---- few long requests: several workgroups to a KV head, in three launches --------------------------------
// First each counts its part's first digits; then each adds the counts up, finds the digit of the bar, and lists its part's ranks of that digit; then each finds
// the bar from all lists, knows from them how many keys of earlier parts stay, and writes its own.  Where too many ranks share the digit, the first
// workgroup does all of it by itself.  One request of 98304 keys, eight heads: 25.8 us (4.6 + 9.5 + 13.0 one by one in a trace), 65 by one workgroup a head.
constexpr int kPartThreads = 512;

struct Part {
  uint16_t counts[kBins];
  uint32_t list[kKeepPartList];
  int above, listed, digit, higher;                      // keys above the bar's digit, and of it, in this part; the digit, and keys above it in the whole request
};
static_assert(sizeof(Part) == kKeepPartBytes, "");

struct Range {
  int from, to;
};
__device__ inline Range part_of(const PageKeepArgs& a, int len, int part) {
  const int each = ((len + a.parts - 1) / a.parts + 255) & ~255, from = min(part * each, len);
  return Range{from, min(from + each, len)};
}

template <int STEP>
__global__ __launch_bounds__(kPartThreads) void page_keep_parts_kernel(const PageKeepArgs a) {
  __shared__ __align__(16) Counts counts;
  __shared__ uint32_t list[STEP == 2 ? kList : 1];
  __shared__ int sums[2];
  const int row = blockIdx.x / a.parts, part = blockIdx.x - row * a.parts, b = row / a.heads, g = row - b * a.heads;
  Part* const parts = reinterpret_cast<Part*>(a.workspace) + (int64_t)row * a.parts;
  const Row r = row_of(a, b, g);
  if (STEP == 2 && part == 0) {
    if (a.lengths_out && g == 0 && threadIdx.x == 0) a.lengths_out[b] = r.stay;
    fill_behind<kPartThreads>(a, r);
  }
  if (r.stay == r.len || (STEP < 2 && r.want == 0)) return;
  const Range own = part_of(a, r.len, part);
  Ranks held;
  load_ranks(a, r, own.from + kWaveKeys * my_wave(), own.to, held);
  if constexpr (STEP == 0) {
    clear<kPartThreads>(counts, kBins);
    each_rank<kPartThreads>(a, r, own.from, own.to, held, [&](uint32_t rank) { count(counts, rank >> 21); });
    __syncthreads();
    for (int d = threadIdx.x; d < kBins; d += kPartThreads) parts[part].counts[d] = (uint16_t)all_copies(counts, d);
  } else if constexpr (STEP == 1) {
    if (threadIdx.x < 2) sums[threadIdx.x] = 0;
    static_assert(kBins == 4 * kPartThreads, "");
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    u16x4 theirs[kKeepMostParts];
#pragma unroll
    for (int p = 0; p < kKeepMostParts; ++p) {
      theirs[p] = u16x4{0, 0, 0, 0};
      if (p < a.parts) theirs[p] = *reinterpret_cast<const u16x4*>(parts[p].counts + kBins - 4 - 4 * threadIdx.x);
    }
    int n[4] = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < kKeepMostParts; ++p)
#pragma unroll
      for (int d = 0; d < 4; ++d) n[d] += theirs[p][3 - d];
    find_digit<kPartThreads>(counts, kBins, r.want, n);
    const uint32_t digit = (uint32_t)counts.found[0];
    int above = 0;
    each_rank<kPartThreads>(a, r, own.from, own.to, held, [&](uint32_t rank) {
      above += rank >> 21 > digit;
      if (rank >> 21 == digit) {
        const int at = atomicAdd(&sums[1], 1);
        if (at < kKeepPartList) parts[part].list[at] = rank;
      }
    });
    if (above) atomicAdd(&sums[0], above);
    __syncthreads();
    if (threadIdx.x == 0) {
      parts[part].above = sums[0];
      parts[part].listed = sums[1];
      parts[part].digit = (int)digit;
      parts[part].higher = counts.found[1];
    }
  } else {
    uint32_t bar = 0;
    int want = r.want, taken = min(own.from, r.first) + max(own.from - r.last, 0), ties = 0;
    if (want > 0) {
      // (a lane has what one of the parts says)
      const int lane = threadIdx.x & 63;
      int listed = 0, above = 0;
      if (lane < a.parts) {
        listed = parts[lane].listed;
        above = parts[lane].above;
      }
      const bool room = !__any(listed > kKeepPartList);
      const int upto = wave_prefix(listed), all = __builtin_amdgcn_readlane(upto, 63), before = __builtin_amdgcn_readlane(upto - listed, part);
      taken += __builtin_amdgcn_readlane(wave_prefix(above) - above, part);
      if (!room || all > kList) {
        if (part > 0) return;
        load_ranks(a, r, kWaveKeys * my_wave(), r.len, held);
        find_bar<kPartThreads>(a, r, counts, list, held, bar, want);
        write_kept<kPartThreads>(a, r, counts, 0, r.len, held, bar, want, 0, 0);
        return;
      }
      for (int p = my_wave(); p < a.parts; p += kPartThreads / 64) {
        const int n = __builtin_amdgcn_readlane(listed, p), at = __builtin_amdgcn_readlane(upto - listed, p);
        for (int i = lane; i < n; i += 64) list[at + i] = parts[p].list[i];
      }
      if (threadIdx.x < 2) sums[threadIdx.x] = 0;
      bar = (uint32_t)parts[0].digit << 21;
      want -= parts[0].higher;
      __syncthreads();
      lower_digits<kPartThreads>(counts, list, all, bar, want);
      int higher = 0, same = 0;
      for (int i = threadIdx.x; i < before; i += kPartThreads) {
        higher += list[i] > bar;
        same += list[i] == bar;
      }
      if (higher) atomicAdd(&sums[0], higher);
      if (same) atomicAdd(&sums[1], same);
      __syncthreads();
      taken += sums[0];
      ties = sums[1];
    }
    write_kept<kPartThreads>(a, r, counts, own.from, own.to, held, bar, want, taken, ties);
  }
}

// Lengths that are written where lengths or budgets are read: in a launch of their own behind all workgroups that read them.
__global__ __launch_bounds__(256) void page_keep_lengths_kernel(const PageKeepArgs a, int* out) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b < a.batch) out[b] = size_of(a, b).stay;
}

}  // namespace

hipError_t launch_page_keep(const PageKeepArgs& args, int64_t rows, hipStream_t s) {
  PageKeepArgs a = args;
  const bool in_place = a.lengths_out == a.lengths || a.lengths_out == a.budgets;
  if (in_place) a.lengths_out = nullptr;
  if (a.parts > 1) {
    const unsigned n = (unsigned)(rows * a.parts);
    page_keep_parts_kernel<0><<<n, kPartThreads, 0, s>>>(a);
    page_keep_parts_kernel<1><<<n, kPartThreads, 0, s>>>(a);
    page_keep_parts_kernel<2><<<n, kPartThreads, 0, s>>>(a);
  } else if (a.max_len <= kKeepShort) {
    page_keep_kernel<512><<<(unsigned)rows, 512, 0, s>>>(a);
  } else {
    page_keep_kernel<1024><<<(unsigned)rows, 1024, 0, s>>>(a);
  }
  if (in_place) page_keep_lengths_kernel<<<(unsigned)((a.batch + 255) / 256), 256, 0, s>>>(a, args.lengths_out);
  return hipGetLastError();
}

}  // namespace mp
