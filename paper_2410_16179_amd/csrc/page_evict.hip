// Keys that stay move to the front of their request's pages, in place, and the pages behind them go back on the free stack.
#include "paged_device.h"

namespace mp {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kUnroll = 4;

__device__ inline int pages_of(int keys, int shift) { return (int)(((int64_t)keys + (1 << shift) - 1) >> shift); }

// Whether the arguments fit, by one workgroup; pages: those that go back.
__device__ inline bool all_fits(const PageEvictArgs& a, int n_free, int64_t& pages) {
  __shared__ int64_t sums[kWaves];
  int64_t sum = 0;
  bool bad = false;
  for (int b = threadIdx.x; b < a.batch; b += kThreads) {
    const int len = a.lengths[b], stay = a.stay[b];
    const bool fits = len >= 0 && len <= a.max_len && stay >= 0 && stay <= len && !(a.kept && stay < len && stay > a.max_keep);
    bad = bad || !fits;
    if (fits) sum += pages_of(len, a.page_shift) - pages_of(stay, a.page_shift);
  }
#pragma unroll
  for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  bad = __syncthreads_or(bad);
  pages = 0;
  for (int w = 0; w < kWaves; ++w) pages += sums[w];
  return !bad && n_free >= 0 && n_free + pages <= a.n_pages;
}

// The pages behind the keys that stay are laid on the stack, requests in order, pages in order.
__device__ inline void give_back(const PageEvictArgs& a, int n_free, bool fits, int64_t pages) {
  __shared__ int wave_total[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) {
    *a.status = fits ? 0 : -1;
    *a.n_free_out = fits ? n_free + (int)pages : n_free;
  }
  if (!fits) return;
  int top = n_free;
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int first = 0, count = 0;
    if (b < a.batch) {
      first = pages_of(a.stay[b], a.page_shift);
      count = pages_of(a.lengths[b], a.page_shift) - first;
    }
    const int upto = wave_prefix(count);
    __syncthreads();
    if (lane == 63) wave_total[wave] = upto;
    __syncthreads();
    int at = top + upto - count;
    for (int w = 0; w < kWaves; ++w) {
      at += w < wave ? wave_total[w] : 0;
      top += wave_total[w];
    }
    // a wavefront's requests one after the other, their pages by its lanes
    for (uint64_t todo = __ballot(count > 0); todo; todo &= todo - 1) {
      const int f = __ffsll((unsigned long long)todo) - 1;
      const int n = __builtin_amdgcn_readlane(count, f), to = __builtin_amdgcn_readlane(at, f);
      const int* from = a.table + (int64_t)__builtin_amdgcn_readlane(b, f) * a.max_pages + __builtin_amdgcn_readlane(first, f);
      for (int j = lane; j < n; j += 64) a.free_pages[to + j] = from[j];
    }
  }
}

// A workgroup takes one array (keys, values, their block scales, accounts) of one request and KV head, or a slice of its rows, and goes over the
// keys that stay in order.  Row j comes from row kept[j] >= j: what a tile of rows overwrites are sources of its own rows and of earlier ones,
// never of later ones.  So a tile's rows are read by all of the workgroup before one of them is written, and later tiles may be on their way.
// Loads come back in the order in which they were asked for, so nothing that is needed at once is asked for behind a tile's rows: page ids come from LDS, the
// list of the tile after next before the next one's rows; and all loads are made by all lanes (those without a row read the first one), so that their number is known.
// (Where a page's rows begin is multiplied out once for each page: for each row it took longer than the rows did.)
// Bound by memory: 32 requests of up to 4160 keys back to 4096 (e4m3, 537 MB moved) 129 us, 4.2 TB/s (154 with page ids asked for behind the rows); one request's
// 32768 keys to 8192 (67 MB) 30.4 to 32.8 us over cards, 2.0 to 2.2 TB/s: rows of 256 bytes in slices of 32, or too few workgroups would be at it (whole rows 103 us).
constexpr int kTable = 4096;                               // pages in LDS; longer requests look in memory
template <class Part>
__device__ inline void move_rows(const PageEvictArgs& a, const PagedArray& r, int b, int g, int64_t slice, int64_t* pages) {
  constexpr int kPart = sizeof(Part);
  const int len = a.lengths[b], stay = a.stay[b], held = pages_of(len, a.page_shift), mask = (1 << a.page_shift) - 1;
  if (stay == 0) return;
  const int* const kept = a.kept + ((int64_t)b * a.heads + g) * a.max_keep;
  const int* const table = a.table + (int64_t)b * a.max_pages;
  const uint32_t key_bytes = (uint32_t)r.key;
  const bool near = held <= kTable;
  __syncthreads();                                         // (the last request's are done with)
  auto page_at = [&](int i) {                              // -1: there is none
    const int id = table[i];
    return (uint32_t)id < (uint32_t)a.n_pages ? id * r.page : (int64_t)-1;
  };
  if (near)
    for (int i = threadIdx.x; i < held; i += kThreads) pages[i] = page_at(i);
  const int lanes = r.slice / kPart, step = kThreads / lanes, row0 = threadIdx.x / lanes, tile = step * kUnroll;
  char* const base = r.at + g * r.head + slice * r.slice + (threadIdx.x - row0 * lanes) * kPart;
  // the first key that moves: kept[j] == j up to it, and nowhere behind
  int lo = 0, hi = stay;
  while (lo < hi) {
    const int lane = threadIdx.x & 63, each = (hi - lo + 63) / 64, j = lo + lane * each;
    const uint64_t moved = __ballot(j >= hi || kept[j] != j);
    const int f = moved ? __ffsll((unsigned long long)moved) - 1 : 64;
    if (f == 0) break;
    const int low = lo + (f - 1) * each + 1;
    hi = min(hi, lo + f * each);
    lo = low;
  }
  __syncthreads();
  // where a key's row is; a key on a page that is none has none
  auto place = [&](int key, bool& there) -> char* {
    const int64_t page = near ? pages[key >> a.page_shift] : page_at(key >> a.page_shift);
    there = page >= 0;
    return base + (there ? page : 0) + (uint32_t)(key & mask) * key_bytes;   // (below 2^31 within a page)
  };
  // three steps in flight: a tile's list, its rows, its writing
  Part now[kUnroll], next[kUnroll];
  int from[kUnroll], after[kUnroll];
  auto list = [&](int j0, int (&to)[kUnroll]) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) to[i] = kept[min(j0 + row0 + i * step, stay - 1)];
  };
  auto fetch = [&](int j0, Part (&to)[kUnroll]) {
    uint32_t moves = 0;
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int j = j0 + row0 + i * step;
      bool there;
      const bool real = j < stay && from[i] > j && from[i] < len;
      const char* src = place(real ? from[i] : 0, there);
      to[i] = *reinterpret_cast<const Part*>(src);
      moves |= real && there ? 1u << i : 0u;
    }
    return moves;
  };
  int j0 = __builtin_amdgcn_readfirstlane(lo);
  list(j0, from);
  list(j0 + tile, after);
  uint32_t here = fetch(j0, now);
#pragma unroll 1
  for (; j0 < stay; j0 += tile) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) from[i] = after[i];
    list(j0 + 2 * tile, after);
    const uint32_t ahead = fetch(j0 + tile, next);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) asm volatile("" : "+v"(now[i]));   // (read before the barrier)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      bool there = false;
      char* to = nullptr;
      if (here >> i & 1) to = place(j0 + row0 + i * step, there);
      if (there) *reinterpret_cast<Part*>(to) = now[i];
      now[i] = next[i];
    }
    here = ahead;
  }
}

// Workgroups that move rows, and one that keeps the books, the first (`books` 1); each looks at the arguments for itself, so the stack's height must not
// change meanwhile: where it is written in place the books come in a launch of their own (no job is left for the others).
__global__ __launch_bounds__(kThreads) void page_evict_kernel(const PageEvictArgs a, int jobs, int books) {
  const int n_free = *a.n_free;
  int64_t pages;
  const bool fits = all_fits(a, n_free, pages);
  if (blockIdx.x < books) {
    give_back(a, n_free, fits, pages);
    return;
  }
  if (!fits) return;
  __shared__ int64_t pages_at[kTable];
  const int64_t units = (int64_t)a.batch * a.heads, all = units * jobs;
#pragma unroll 1
  for (int64_t n = (int64_t)blockIdx.x - books; n < all; n += gridDim.x - books) {
    int job = (int)(n / units), array = 0;                 // (the slices of a unit's rows, which share lines, on one XCD where units go with eight)
    const int64_t unit = n - job * units;
    const int b = (int)(unit / a.heads), g = (int)(unit - (int64_t)b * a.heads);
    if (a.stay[b] == a.lengths[b]) continue;
    while (job >= a.arrays[array].slices) job -= a.arrays[array++].slices;
    const PagedArray r = a.arrays[array];
    if (r.slice == 4) move_rows<uint32_t>(a, r, b, g, job, pages_at);
    else move_rows<u32x4>(a, r, b, g, job, pages_at);
  }
}

}  // namespace

hipError_t launch_page_evict(const PageEvictArgs& a, hipStream_t s) {
  int jobs = 0;
  if (a.kept)
    for (const PagedArray& r : a.arrays) jobs += r.slices;
  const int64_t all = (int64_t)a.batch * a.heads * jobs, most = 65535;
  const unsigned movers = (unsigned)(all < most ? all : most);
  const bool in_place = a.n_free == a.n_free_out;
  if (movers > 0) page_evict_kernel<<<movers + !in_place, kThreads, 0, s>>>(a, jobs, !in_place);
  if (movers == 0 || in_place) page_evict_kernel<<<1, kThreads, 0, s>>>(a, 1, 1);
  return hipGetLastError();
}

}  // namespace mp
