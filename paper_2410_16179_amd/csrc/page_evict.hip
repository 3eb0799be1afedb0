// Keys that stay move to the front of their request's pages, in place, and the pages behind them go back on the free stack.
#include "paged_device.h"

namespace mp {
namespace {

constexpr int kThreads = 512, kUnroll = 4;

__device__ inline int pages_of(int keys, int shift) { return (int)(((int64_t)keys + (1 << shift) - 1) >> shift); }

// One workgroup: what is asked for is looked at, and the pages behind the keys that stay are laid on the stack, requests in order, pages in order.
constexpr int kBookThreads = 1024;
__global__ __launch_bounds__(kBookThreads) void page_evict_book_kernel(const PageEvictArgs a) {
  __shared__ int64_t total;
  __shared__ int wrong, wave_total[kBookThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) { total = 0; wrong = 0; }
  __syncthreads();
  const int n_free = *a.n_free;
  int64_t sum = 0;
  bool bad = false;
  for (int b = threadIdx.x; b < a.batch; b += kBookThreads) {
    const int len = a.lengths[b], stay = a.stay[b];
    bad = bad || len < 0 || len > a.max_len || stay < 0 || stay > len || (a.kept && stay < len && stay > a.max_keep);
    if (!bad) sum += pages_of(len, a.page_shift) - pages_of(stay, a.page_shift);
  }
  if (bad) atomicOr(&wrong, 1);
  atomicAdd(reinterpret_cast<unsigned long long*>(&total), (unsigned long long)sum);
  __syncthreads();
  const bool fine = !wrong && n_free >= 0 && n_free + total <= a.n_pages;
  if (threadIdx.x == 0) {
    *a.status = fine ? 0 : -1;
    *a.n_free_out = fine ? n_free + (int)total : n_free;
  }
  if (!fine) return;
  int top = n_free;
  for (int b0 = 0; b0 < a.batch; b0 += kBookThreads) {
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
    for (int w = 0; w < kBookThreads / 64; ++w) {
      at += w < wave ? wave_total[w] : 0;
      top += wave_total[w];
    }
    for (int j = 0; j < count; ++j) a.free_pages[at + j] = a.table[(int64_t)b * a.max_pages + first + j];
  }
}

// A workgroup takes one array (keys, values, their block scales, accounts) of one request and KV head, or a slice of its rows, and goes over the
// keys that stay in order.  Row j comes from row kept[j] >= j: what a tile of rows overwrites are sources of its own rows and of earlier ones,
// never of later ones.  So a tile's rows are read by all of the workgroup before one of them is written, and later tiles may be on their way.
template <class Part>
__device__ inline void move_rows(const PageEvictArgs& a, const PagedArray& r, int b, int g, int64_t slice) {
  constexpr int kPart = sizeof(Part);
  const int len = a.lengths[b], stay = a.stay[b];
  const int* const kept = a.kept + ((int64_t)b * a.heads + g) * a.max_keep;
  const int* const table = a.table + (int64_t)b * a.max_pages;
  const int lanes = r.slice / kPart, step = kThreads / lanes, row0 = threadIdx.x / lanes, tile = step * kUnroll;
  char* const base = r.at + g * r.head + slice * r.slice + (threadIdx.x - row0 * lanes) * kPart;
  auto place = [&](int key) -> char* {
    const int id = table[key >> a.page_shift];
    return (uint32_t)id < (uint32_t)a.n_pages ? base + id * r.page + (key & ((1 << a.page_shift) - 1)) * r.key : nullptr;
  };
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
  Part now[kUnroll], next[kUnroll];
  auto fetch = [&](int j0, Part (&to)[kUnroll], bool (&there)[kUnroll]) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int j = j0 + row0 + i * step, from = j < stay ? kept[j] : -1;
      const char* src = from > j && from < len ? place(from) : nullptr;
      there[i] = src != nullptr;
      if (src) to[i] = *reinterpret_cast<const Part*>(src);
    }
  };
  bool here[kUnroll], ahead[kUnroll];
  int j0 = __builtin_amdgcn_readfirstlane(lo);
  fetch(j0, now, here);
#pragma unroll 1
  for (; j0 < stay; j0 += tile) {
    fetch(j0 + tile, next, ahead);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) asm volatile("" : "+v"(now[i]));   // (read before the barrier)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      char* to = here[i] ? place(j0 + row0 + i * step) : nullptr;
      if (to) *reinterpret_cast<Part*>(to) = now[i];
      now[i] = next[i];
      here[i] = ahead[i];
    }
  }
}

__global__ __launch_bounds__(kThreads) void page_evict_move_kernel(const PageEvictArgs a) {
  if (*a.status != 0) return;
  const int64_t units = (int64_t)a.batch * a.heads;
  int job = blockIdx.x, array = 0;
  while (job >= a.arrays[array].slices) job -= a.arrays[array++].slices;
  const PagedArray r = a.arrays[array];
#pragma unroll 1
  for (int64_t unit = blockIdx.y; unit < units; unit += gridDim.y) {
    const int b = (int)(unit / a.heads), g = (int)(unit - (int64_t)b * a.heads);
    if (a.stay[b] == a.lengths[b]) continue;
    if (r.slice == 4) move_rows<uint32_t>(a, r, b, g, job);
    else move_rows<u32x4>(a, r, b, g, job);
  }
}

}  // namespace

hipError_t launch_page_evict(const PageEvictArgs& a, hipStream_t s) {
  page_evict_book_kernel<<<1, kBookThreads, 0, s>>>(a);
  int jobs = 0;
  for (const PagedArray& r : a.arrays) jobs += r.slices;
  const int64_t units = (int64_t)a.batch * a.heads;
  if (a.kept && units > 0 && jobs > 0)
    page_evict_move_kernel<<<dim3((unsigned)jobs, (unsigned)(units < 65535 ? units : 65535)), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mp
