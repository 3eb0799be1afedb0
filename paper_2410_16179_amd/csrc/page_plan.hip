// One step's bookkeeping of a paged cache: pages handed out and taken back, block tables, slots.
//
// Three sums over the requests decide everything: new tokens (where a request's rows begin), pages that requests need, and pages
// that ended requests give back.  The stack of free pages with the ended requests' pages on top is never formed: entry x of it
// is looked up where it lies, in the stack or in an ended request's table row, and page k handed out is entry height - 1 - k.
// A slot then follows from a token's row alone.  Bound by latency: a few thousand bytes, read in three dependent steps
// (requests, table entry or stack entry, and for tokens behind a request's first the search for their request).  64 requests of
// one token 2.9 us, 512 with 35840 token rows 5.7 (345 KB); a kernel that does nothing takes 2.
#include "paged_common.h"

namespace mp {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanLds = kPlanInOneRequests;   // requests whose prefix sums are kept in LDS

// Sums that stop at 2^32 - 1: whatever the device memory holds, a sum that is too large stays too large.
__device__ inline uint32_t add(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
template <int CTRL, int ROWS>
__device__ inline uint32_t plan_lane(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, ROWS == 0xf);
}
__device__ inline uint32_t plan_row_prefix(uint32_t v) {   // inclusive, over rows of sixteen lanes
  v = add(v, plan_lane<0x111, 0xf>(v));
  v = add(v, plan_lane<0x112, 0xf>(v));
  v = add(v, plan_lane<0x114, 0xf>(v));
  return add(v, plan_lane<0x118, 0xf>(v));
}
__device__ inline uint32_t plan_prefix(uint32_t v) {       // inclusive, over the wavefront
  v = plan_row_prefix(v);
  v = add(v, plan_lane<0x142, 0xa>(v));
  return add(v, plan_lane<0x143, 0xc>(v));
}

struct PlanSum { uint32_t tokens, need, back; };
__device__ inline PlanSum operator+(const PlanSum& x, const PlanSum& y) { return {add(x.tokens, y.tokens), add(x.need, y.need), add(x.back, y.back)}; }

struct PlanTotals { int n_free, tokens, need, back, status; };

// Sums over the threads before this one; `all` gets the total.
__device__ inline PlanSum block_prefix(const PlanSum& v, PlanSum* lds, PlanSum& all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PlanSum upto{plan_prefix(v.tokens), plan_prefix(v.need), plan_prefix(v.back)};
  if (lane == 63) lds[wave] = upto;
  __syncthreads();
  const PlanSum w = lds[lane & 15];                         // (sixteen wavefronts)
  const PlanSum waves{plan_row_prefix(w.tokens), plan_row_prefix(w.need), plan_row_prefix(w.back)};
  auto at = [&](uint32_t x, int l) { return (uint32_t)__builtin_amdgcn_readlane((int)x, l); };
  all = {at(waves.tokens, 15), at(waves.need, 15), at(waves.back, 15)};
  PlanSum before{0, 0, 0};
  if (wave > 0) before = {at(waves.tokens, wave - 1), at(waves.need, wave - 1), at(waves.back, wave - 1)};
  __syncthreads();
  return before + PlanSum{upto.tokens - v.tokens, upto.need - v.need, upto.back - v.back};   // (a sum that has stopped: not used)
}

// Reads every request, leaves the sums over the requests before it (and the totals behind the last) in t0, a0, r0 and, if asked
// for, its length; works out the status.  Run by one whole workgroup.  With a status other than 0 the sums mean nothing.
// singles: whether no request has more than one new token.
__device__ inline PlanTotals plan_sums(const PagePlanArgs& a, int* t0, int* a0, int* r0, int* length, bool& singles) {
  static_assert(kPlanThreads == 16 * 64, "block_prefix takes sixteen wavefronts");
  __shared__ PlanSum lds[kPlanThreads / 64];
  __shared__ int flags;
  if (threadIdx.x == 0) flags = 0;
  PlanSum carry{0, 0, 0};
  bool wrong = false, several = false;
  const int page = 1 << a.page_shift;
  const int64_t room = (int64_t)a.max_pages << a.page_shift;
  PlanTotals t;
  t.n_free = *a.n_free;
  for (int b0 = 0; b0 < a.batch; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    PlanSum v{0, 0, 0};
    int len = 0;
    if (b < a.batch) {
      const int n = a.new_tokens[b];
      len = a.lengths[b];
      const bool bad = n < -1 || n > a.max_new || len < 0 || (int64_t)len + (n > 0 ? n : 0) > room;
      wrong = wrong || bad;
      several = several || n > 1;
      if (!bad) {
        const uint32_t held = (uint32_t)(len + page - 1) >> a.page_shift;
        if (n < 0) v.back = held;
        else { v.tokens = n; v.need = ((uint32_t)(len + n + page - 1) >> a.page_shift) - held; }
      }
    }
    PlanSum all;
    const PlanSum before = carry + block_prefix(v, lds, all);
    if (b < a.batch) {
      t0[b] = (int)before.tokens;
      a0[b] = (int)before.need;
      r0[b] = (int)before.back;
      if (length) length[b] = len;
    }
    carry = carry + all;
  }
  if (threadIdx.x == 0) { t0[a.batch] = (int)carry.tokens; a0[a.batch] = (int)carry.need; r0[a.batch] = (int)carry.back; }
  wrong = wrong || carry.tokens > a.max_tokens || t.n_free < 0 || (int64_t)t.n_free + carry.back > a.n_pages;
  const int mine = (__any(wrong) ? 1 : 0) | (__any(several) ? 2 : 0);
  if (a.batch == 0) __syncthreads();                       // (flags are 0; otherwise behind the barriers of the sums)
  if (mine && (threadIdx.x & 63) == 0) atomicOr(&flags, mine);
  __syncthreads();
  const int64_t missing = (int64_t)carry.need - t.n_free - carry.back;
  t.status = flags & 1 ? -1 : (missing > 0 ? (int)(missing < INT32_MAX ? missing : INT32_MAX) : 0);
  singles = !(flags & 2);
  t.tokens = (int)carry.tokens;
  t.need = (int)carry.need;
  t.back = (int)carry.back;
  return t;
}

// What is known of every request, by one workgroup.
__device__ inline void plan_requests(const PagePlanArgs& a, const PlanTotals& t, const int* t0) {
  for (int b = threadIdx.x; b < a.batch; b += kPlanThreads) {
    const int n = a.new_tokens[b], len = a.lengths[b];
    a.lengths_out[b] = t.status ? len : (n < 0 ? 0 : len + n);
    a.token_start[b] = t.status ? 0 : t0[b];
  }
  if (threadIdx.x == 0) {
    a.token_start[a.batch] = t.status ? 0 : t.tokens;
    *a.status = t.status;
    *a.n_free_out = t.status ? t.n_free : t.n_free + t.back - t.need;
  }
}

// Last request whose sum is at most i (sums are ascending, first 0; i is below the total).
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

// Slot of the token at position pos of request b.  A page that is handed out is entered into the table by the one token that opens it.
// Entries of the stack below its old height are only read and rows of ended requests too, and entries of pages held before, so no
// thread writes what another reads.
__device__ inline int64_t plan_slot(const PagePlanArgs& a, const PlanTotals& t, const int* r0, int b, int len, int pos, int opened) {
  const int page = 1 << a.page_shift, held = (len + page - 1) >> a.page_shift, p = pos >> a.page_shift;
  int* entry = a.table + (int64_t)b * a.max_pages + p;
  int id;
  if (p < held) {
    id = *entry;
  } else {
    id = plan_stack(a, t, r0, t.n_free + t.back - 1 - (opened + p - held));
    if ((pos & (page - 1)) == 0) *entry = id;
  }
  return (int64_t)id * page + (pos & (page - 1));
}

// Slots of the rows first, first + step, .., and the stack's new entries.
template <class Length>
__device__ inline void plan_fill(const PagePlanArgs& a, const PlanTotals& t, const int* t0, const int* a0, const int* r0, Length length, int64_t first,
                                 int64_t step) {
  const int64_t left = t.status ? 0 : (t.back > t.need ? t.back - t.need : 0);
  const int64_t most = a.max_tokens > left ? a.max_tokens : left;
  for (int64_t i = first; i < most; i += step) {
    if (i < a.max_tokens) {
      int64_t slot = -1;
      if (!t.status && i < t.tokens) {
        const int b = plan_owner(t0, a.batch, (int)i), len = length(b);
        slot = plan_slot(a, t, r0, b, len, len + (int)i - t0[b], a0[b]);
      }
      a.slots[i] = slot;
    }
    if (i < left) a.free_pages[t.n_free + i] = plan_stack(a, t, r0, t.n_free + (int)i);
  }
}

// Everything in one launch, the sums in LDS.  Several workgroups all work out the sums, the first one writes what is known of the requests, and
// each takes its rows; they read what `lengths` and n_free hold, so these are not lengths_out and n_free_out then.
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(const PagePlanArgs a) {
  __shared__ int t0[kPlanLds + 1], a0[kPlanLds + 1], r0[kPlanLds + 1], len[kPlanLds];
  bool singles;
  const PlanTotals t = plan_sums(a, t0, a0, r0, len, singles);
  if (gridDim.x == 1 && singles) {
    // one token a request at most: no search for a row's request
    const int64_t left = t.status ? 0 : (t.back > t.need ? t.back - t.need : 0);
    for (int b = threadIdx.x; b < a.batch; b += kPlanThreads)
      if (!t.status && t0[b + 1] > t0[b]) a.slots[t0[b]] = plan_slot(a, t, r0, b, len[b], len[b], a0[b]);
    for (int64_t i = (t.status ? 0 : t.tokens) + (int64_t)threadIdx.x; i < a.max_tokens; i += kPlanThreads) a.slots[i] = -1;
    for (int64_t i = threadIdx.x; i < left; i += kPlanThreads) a.free_pages[t.n_free + i] = plan_stack(a, t, r0, t.n_free + (int)i);
    plan_requests(a, t, t0);
    return;
  }
  if (blockIdx.x == 0) plan_requests(a, t, t0);
  plan_fill(a, t, t0, a0, r0, [&](int b) { return len[b]; }, (int64_t)blockIdx.x * kPlanThreads + threadIdx.x, (int64_t)gridDim.x * kPlanThreads);
}

// In two launches: one workgroup leaves the sums in the workspace, all of the chip fills in the slots.
__global__ __launch_bounds__(kPlanThreads) void page_plan_sums_kernel(const PagePlanArgs a) {
  int* t0 = a.scan;
  bool singles;
  const PlanTotals t = plan_sums(a, t0, t0 + a.batch + 1, t0 + 2 * (a.batch + 1), nullptr, singles);
  plan_requests(a, t, t0);
}
template <bool LDS>
__global__ __launch_bounds__(256) void page_plan_fill_kernel(const PagePlanArgs a) {
  const int *t0 = a.scan, *a0 = t0 + a.batch + 1, *r0 = a0 + a.batch + 1;
  __shared__ int sums[LDS ? 3 * (kPlanLds + 1) : 1];
  if (LDS) {
    for (int i = threadIdx.x; i < 3 * (a.batch + 1); i += 256) sums[i] = a.scan[i];
    __syncthreads();
    t0 = sums; a0 = t0 + a.batch + 1; r0 = a0 + a.batch + 1;
  }
  PlanTotals t;
  t.status = *a.status;
  t.tokens = t0[a.batch]; t.need = a0[a.batch]; t.back = r0[a.batch];
  t.n_free = *a.n_free_out - t.back + t.need;              // (n_free may be the same word)
  plan_fill(a, t, t0, a0, r0, [&](int b) { return a.lengths_out[b] - (t0[b + 1] - t0[b]); },
            (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t s) {
  const bool in_place = a.lengths_out == a.lengths || a.n_free_out == a.n_free;
  const int one = page_plan_workgroups(a.batch, a.max_tokens, in_place);
  if (one > 0) {
    page_plan_kernel<<<one, kPlanThreads, 0, s>>>(a);
  } else {
    // (pages that come back may be more than the tokens: the loop goes on for them)
    const int64_t blocks = (a.max_tokens + 255) / 256, most = 16 * kNumCU;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    page_plan_sums_kernel<<<1, kPlanThreads, 0, s>>>(a);
    if (a.batch <= kPlanLds) page_plan_fill_kernel<true><<<grid, 256, 0, s>>>(a);
    else page_plan_fill_kernel<false><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace mp
