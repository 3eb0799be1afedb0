// One step's bookkeeping of a paged cache: pages handed out and taken back, block tables, slots.
#include "paged_common.h"

namespace mp {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanLds = kPlanInOneRequests;   // requests whose prefix sums are kept in LDS

// Three sums over the requests: new tokens, pages that they need, pages that ended requests give back.
struct PlanSum { int64_t tokens, need, back; };
__device__ inline PlanSum operator+(const PlanSum& x, const PlanSum& y) { return {x.tokens + y.tokens, x.need + y.need, x.back + y.back}; }
__device__ inline PlanSum shuffled_up(const PlanSum& v, int d) {
  return {(int64_t)__shfl_up((long long)v.tokens, d), (int64_t)__shfl_up((long long)v.need, d), (int64_t)__shfl_up((long long)v.back, d)};
}

struct PlanTotals { int n_free; int tokens, need, back; int status; };

// Inclusive prefix sums over the workgroup's threads; `all` gets the total.
__device__ inline PlanSum block_prefix(PlanSum v, PlanSum* lds, PlanSum& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const PlanSum u = shuffled_up(v, d);
    if (lane >= d) v = v + u;
  }
  if (lane == 63) lds[wave] = v;
  __syncthreads();
  PlanSum before{0, 0, 0};
  all = {0, 0, 0};
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before = before + lds[w];
    all = all + lds[w];
  }
  __syncthreads();
  return before + v;
}

// Reads every request, leaves the exclusive prefix sums (and the totals behind the last) in t0, a0, r0, and works out
// the status.  Run by one whole workgroup.  With a status other than 0 the sums mean nothing.
__device__ inline PlanTotals plan_sums(const PagePlanArgs& a, int* t0, int* a0, int* r0) {
  __shared__ PlanSum lds[kPlanThreads / 64];
  PlanSum carry{0, 0, 0};
  bool wrong = false;
  const int page = 1 << a.page_shift;
  const int64_t room = (int64_t)a.max_pages << a.page_shift;
  for (int b0 = 0; b0 < a.batch; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    PlanSum v{0, 0, 0};
    if (b < a.batch) {
      const int64_t n = a.new_tokens[b], len = a.lengths[b];
      const bool ended = n < 0;
      const int64_t held = (len + page - 1) >> a.page_shift;
      wrong = wrong || n < -1 || n > a.max_new || len < 0 || len + (ended ? 0 : n) > room;
      if (ended) v.back = held;
      else { v.tokens = n; v.need = ((len + n + page - 1) >> a.page_shift) - held; }
    }
    PlanSum all;
    const PlanSum upto = carry + block_prefix(v, lds, all);
    if (b < a.batch) {
      t0[b] = (int)(upto.tokens - v.tokens);
      a0[b] = (int)(upto.need - v.need);
      r0[b] = (int)(upto.back - v.back);
    }
    carry = carry + all;
  }
  if (threadIdx.x == 0) { t0[a.batch] = (int)carry.tokens; a0[a.batch] = (int)carry.need; r0[a.batch] = (int)carry.back; }
  PlanTotals t;
  t.n_free = *a.n_free;
  wrong = wrong || carry.tokens > a.max_tokens || t.n_free < 0 || t.n_free + carry.back > a.n_pages;
  const bool bad = __syncthreads_or(wrong);
  const int64_t missing = carry.need - t.n_free - carry.back;
  t.status = bad ? -1 : (missing > 0 ? (int)(missing < INT32_MAX ? missing : INT32_MAX) : 0);
  t.tokens = (int)carry.tokens;
  t.need = (int)carry.need;
  t.back = (int)carry.back;
  return t;
}

// What is known of every request, by one workgroup.
__device__ inline void plan_requests(const PagePlanArgs& a, const PlanTotals& t, const int* t0, int* old_len) {
  for (int b = threadIdx.x; b < a.batch; b += kPlanThreads) {
    const int n = a.new_tokens[b], len = a.lengths[b];
    if (old_len) old_len[b] = len;
    a.lengths_out[b] = t.status ? len : (n < 0 ? 0 : len + n);
    a.token_start[b] = t.status ? 0 : t0[b];
  }
  if (threadIdx.x == 0) {
    a.token_start[a.batch] = t.status ? 0 : t.tokens;
    *a.status = t.status;
    *a.n_free_out = t.status ? t.n_free : t.n_free + t.back - t.need;
  }
}

// Last request whose prefix sum is at most i (sums are ascending, first 0; i is below the last).
__device__ inline int plan_owner(const int* sums, int batch, int i) {
  int lo = 0, hi = batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Entry x of the stack: what it held, and on top of that the pages of the ended requests.
__device__ inline int plan_stack(const PagePlanArgs& a, const PlanTotals& t, const int* r0, int x) {
  if (x < t.n_free) return a.free_pages[x];
  const int r = x - t.n_free, b = plan_owner(r0, a.batch, r);
  return a.table[(int64_t)b * a.max_pages + (r - r0[b])];
}

// Slots of all tokens, and the table's and the stack's new entries.  A page that is handed out is entered into the
// table by the one token that opens it.  Entries of the stack below its old height are only read and rows of
// ended requests too, so no thread writes what another reads.
template <class OldLength>
__device__ inline void plan_fill(const PagePlanArgs& a, const PlanTotals& t, const int* t0, const int* a0, const int* r0, OldLength old_length,
                                 int64_t first, int64_t step) {
  const int page = 1 << a.page_shift;
  const int64_t left = t.status ? 0 : (t.back > t.need ? t.back - t.need : 0);
  const int64_t most = a.max_tokens > left ? a.max_tokens : left;
  for (int64_t i = first; i < most; i += step) {
    if (i < a.max_tokens) {
      int64_t slot = -1;
      if (!t.status && i < t.tokens) {
        const int b = plan_owner(t0, a.batch, (int)i), len = old_length(b);
        const int pos = len + (int)i - t0[b], held = (len + page - 1) >> a.page_shift, p = pos >> a.page_shift;
        int id;
        int* entry = a.table + (int64_t)b * a.max_pages + p;
        if (p < held) {
          id = *entry;
        } else {
          id = plan_stack(a, t, r0, t.n_free + t.back - 1 - (a0[b] + p - held));
          if ((pos & (page - 1)) == 0) *entry = id;
        }
        slot = (int64_t)id * page + (pos & (page - 1));
      }
      a.slots[i] = slot;
    }
    if (i < left) a.free_pages[t.n_free + i] = plan_stack(a, t, r0, t.n_free + (int)i);
  }
}

// Everything in one workgroup, the sums in LDS.
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(const PagePlanArgs a) {
  __shared__ int t0[kPlanLds + 1], a0[kPlanLds + 1], r0[kPlanLds + 1], len[kPlanLds];
  const PlanTotals t = plan_sums(a, t0, a0, r0);
  plan_requests(a, t, t0, len);
  __syncthreads();
  plan_fill(a, t, t0, a0, r0, [&](int b) { return len[b]; }, threadIdx.x, kPlanThreads);
}

// In two launches: one workgroup leaves the sums in the workspace, all of the chip fills in the slots.
__global__ __launch_bounds__(kPlanThreads) void page_plan_sums_kernel(const PagePlanArgs a) {
  int* t0 = a.scan;
  const PlanTotals t = plan_sums(a, t0, t0 + a.batch + 1, t0 + 2 * (a.batch + 1));
  plan_requests(a, t, t0, nullptr);
}
__global__ __launch_bounds__(256) void page_plan_fill_kernel(const PagePlanArgs a) {
  const int *t0 = a.scan, *a0 = t0 + a.batch + 1, *r0 = a0 + a.batch + 1;
  PlanTotals t;
  t.status = *a.status;
  t.tokens = t0[a.batch]; t.need = a0[a.batch]; t.back = r0[a.batch];
  t.n_free = *a.n_free_out - t.back + t.need;              // (n_free may be the same word)
  plan_fill(a, t, t0, a0, r0, [&](int b) { return a.lengths_out[b] - (t0[b + 1] - t0[b]); },
            (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t s) {
  if (page_plan_in_one(a.batch, a.max_tokens)) {
    page_plan_kernel<<<1, kPlanThreads, 0, s>>>(a);
  } else {
    // (pages that come back may be more than the tokens: the loop goes on for them)
    const int64_t blocks = (a.max_tokens + 255) / 256, most = 16 * kNumCU;
    page_plan_sums_kernel<<<1, kPlanThreads, 0, s>>>(a);
    page_plan_fill_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace mp
