// Which keys of a request stay: the first ones, the last ones, and those with the largest accounts.
#include "paged_device.h"

namespace mp {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// The accounts' order as that of unsigned integers: NaN below all, both zeros alike.
__device__ inline uint32_t rank_of(float w) {
  const uint32_t bits = __float_as_uint(w + 0.f);
  const uint32_t up = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
  return w == w ? up : 0u;
}

struct Row {
  const int* table; const float* weights;
  int len, stay, first, last;
};
__device__ inline bool always(const Row& r, int i) { return i < r.first || i >= r.len - r.last; }

// Ranks of keys i .. i + 3 (i a multiple of four); 0 beyond the last one and on pages that are none.
__device__ inline void four_ranks(const PageKeepArgs& a, const Row& r, int i, uint32_t (&rank)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) rank[e] = 0;
  if (i >= r.len) return;
  const int id = r.table[i >> a.page_shift];
  if ((uint32_t)id >= (uint32_t)a.n_pages) return;
  const f32x4 w = *reinterpret_cast<const f32x4*>(r.weights + (((int64_t)id * a.heads) << a.page_shift) + (i & ((1 << a.page_shift) - 1)));
#pragma unroll
  for (int e = 0; e < 4; ++e) rank[e] = i + e < r.len ? rank_of(w[e]) : 0u;
}

// A workgroup per request and KV head.  The smallest rank that stays is found a byte at a time by counting (equal ranks: the first ones stay),
// and then the keys are gone over in order.
__global__ __launch_bounds__(kThreads) void page_keep_kernel(const PageKeepArgs a) {
  __shared__ int bins[256];
  __shared__ int found[2];
  __shared__ int totals[2][kWaves];
  const int b = blockIdx.x / a.heads, g = blockIdx.x - b * a.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int len = a.lengths[b];
  len = len < 0 ? 0 : (len > a.max_len ? a.max_len : len);
  const int budget = a.budgets[b], most = budget < a.max_keep ? budget : a.max_keep;
  const int stay = budget < 0 || len <= most ? len : most;
  int* const kept = a.kept + ((int64_t)b * a.heads + g) * a.max_keep;
  if (g == 0 && threadIdx.x == 0) a.lengths_out[b] = stay;
  if (stay == len) {
    for (int j = threadIdx.x; j < a.max_keep; j += kThreads) kept[j] = -1;
    return;
  }
  const Row r{a.table + (int64_t)b * a.max_pages, a.weights + ((int64_t)g << a.page_shift), len, stay, a.n_first, a.n_last};
  const int64_t both = (int64_t)a.n_first + a.n_last;
  const int sure = both < len ? (int)both : len;
  // keys that are chosen by their accounts: those of rank above `bar`, and the first `equal` ones of that rank
  uint32_t bar = 0xffffffffu;
  int want = stay - sure;
  if (want > 0) {
    bar = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += kThreads) bins[i] = 0;
      __syncthreads();
      for (int i = 4 * threadIdx.x; i < len; i += 4 * kThreads) {
        uint32_t rank[4];
        four_ranks(a, r, i, rank);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (i + e < len && !always(r, i + e) && (shift == 24 || rank[e] >> (shift + 8) == bar >> (shift + 8)))
            atomicAdd(&bins[rank[e] >> shift & 255], 1);
      }
      __syncthreads();
      if (wave == 0) {
        // from the largest byte down: the one at which `want` keys are reached; a lane has four
        int own = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) own += bins[255 - 4 * lane - e];
        const int upto = wave_prefix(own);
        const uint64_t reached = __ballot(upto >= want);
        if (lane == __ffsll((unsigned long long)reached) - 1) {
          int before = upto - own, byte = 255 - 4 * lane;
          while (before + bins[byte] < want) before += bins[byte--];
          found[0] = byte;
          found[1] = before;
        }
      }
      __syncthreads();
      bar |= (uint32_t)found[0] << shift;
      want -= found[1];
      __syncthreads();
    }
  }
  const int equal = want > 0 ? want : 0;                   // (of rank `bar`)
  int out = 0, ties = 0;
#pragma unroll 1
  for (int i0 = 0; i0 < len && out < stay; i0 += 4 * kThreads) {
    const int i = i0 + 4 * threadIdx.x;
    uint32_t rank[4];
    four_ranks(a, r, i, rank);
    int tie[4], same = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      tie[e] = i + e < len && !always(r, i + e) && equal > 0 && rank[e] == bar;
      same += tie[e];
    }
    const int same_upto = wave_prefix(same);
    if (lane == 63) totals[0][wave] = same_upto;
    __syncthreads();
    int rank_of_tie = ties + same_upto - same, all_ties = 0;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const int t = totals[0][x];
      rank_of_tie += x < wave ? t : 0;
      all_ties += t;
    }
    int stays[4], count = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = i + e < len;
      stays[e] = in && (always(r, i + e) || (stay > sure && rank[e] > bar) || (tie[e] && rank_of_tie < equal));
      rank_of_tie += tie[e];
      count += stays[e];
    }
    const int upto = wave_prefix(count);
    if (lane == 63) totals[1][wave] = upto;
    __syncthreads();
    int at = out + upto - count, all = 0;
#pragma unroll
    for (int x = 0; x < kWaves; ++x) {
      const int t = totals[1][x];
      at += x < wave ? t : 0;
      all += t;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (stays[e] && at < stay) kept[at] = i + e;
      at += stays[e];
    }
    out += all;
    ties += all_ties;
  }
  for (int j = stay + threadIdx.x; j < a.max_keep; j += kThreads) kept[j] = -1;
}

}  // namespace

hipError_t launch_page_keep(const PageKeepArgs& a, int64_t rows, hipStream_t s) {
  page_keep_kernel<<<(unsigned)rows, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mp
