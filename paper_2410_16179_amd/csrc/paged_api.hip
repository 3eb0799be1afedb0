// C ABI of the paged cache: argument validation, workspace sizes and kernel launches.  As in magicpig_api.hip,
// validation touches no HIP call.
#include "paged_common.h"

#include <cmath>

namespace {

typedef magicpig_paged_params Params;

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool aligned16(const void* p) { return aligned(p, 16); }
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

constexpr float kLog2e = 1.4426950408889634f;

// new tokens of a request that the token arrays have rows for
int most_new(const Params* p) { return p->max_new < p->max_tokens ? p->max_new : (int)p->max_tokens; }

// what every call looks at
int check(const Params* p) {
  if (!p) return MAGICPIG_INVALID_ARG;
  if (p->batch < 0 || p->n_q_heads <= 0 || p->n_kv_heads <= 0 || p->n_q_heads % p->n_kv_heads != 0) return MAGICPIG_INVALID_ARG;
  if (p->max_pages < 1 || p->n_pages < 1 || p->max_tokens < 1 || p->max_new < 1) return MAGICPIG_INVALID_ARG;
  if (p->n_sink < 0 || p->n_local < 0 || p->n_sink > (1 << 30) || p->n_local > (1 << 30)) return MAGICPIG_INVALID_ARG;
  if (!std::isfinite(p->scale * kLog2e)) return MAGICPIG_INVALID_ARG;
  if (p->head_dim != mp::kHeadDim) return MAGICPIG_UNSUPPORTED;
  if (p->dtype != MAGICPIG_BF16 && p->dtype != MAGICPIG_FP32) return MAGICPIG_UNSUPPORTED;
  if (p->kv_dtype != MAGICPIG_KV_SAME && p->kv_dtype != MAGICPIG_KV_FP8_E4M3 && p->kv_dtype != MAGICPIG_KV_MXFP4) return MAGICPIG_UNSUPPORTED;
  if (p->kv_dtype != MAGICPIG_KV_SAME && p->dtype != MAGICPIG_BF16) return MAGICPIG_UNSUPPORTED;
  if (p->batch > 65536 || p->n_kv_heads > 1024 || p->n_q_heads / p->n_kv_heads > 64) return MAGICPIG_UNSUPPORTED;
  if (p->page_size < 16 || p->page_size > 1024 || (p->page_size & (p->page_size - 1)) != 0) return MAGICPIG_UNSUPPORTED;
  if ((int64_t)p->max_pages * p->page_size > ((int64_t)1 << 30)) return MAGICPIG_UNSUPPORTED;
  if (p->n_pages > INT32_MAX || p->max_tokens > (1 << 24) || p->max_new > (1 << 24)) return MAGICPIG_UNSUPPORTED;
  // workgroups are counted in 32 bits, whatever token counts the device memory holds
  if (mp::paged_most_items(p->batch, p->n_kv_heads, p->n_q_heads / p->n_kv_heads, p->dtype == MAGICPIG_FP32, most_new(p)) > (1 << 30))
    return MAGICPIG_UNSUPPORTED;
  return MAGICPIG_OK;
}

bool four(const Params* p) { return p->kv_dtype == MAGICPIG_KV_MXFP4; }
int64_t row_bytes(const Params* p, int64_t elements) {
  return four(p) ? elements / 2 : elements * (p->kv_dtype == MAGICPIG_KV_FP8_E4M3 ? 1 : (p->dtype == MAGICPIG_FP32 ? 4 : 2));
}

int check_pool(const Params* p, int64_t page, int64_t key, int64_t head) {
  if (page < 0 || key < mp::kHeadDim || head < 0) return MAGICPIG_INVALID_ARG;
  const int64_t unit = four(p) ? mp::kHeadDim : (p->kv_dtype == MAGICPIG_KV_FP8_E4M3 ? 16 : 8);   // (four bits: a row's scales are a word)
  if (page % unit || key % unit || head % unit) return MAGICPIG_UNSUPPORTED;
  if (four(p) && page / unit > UINT32_MAX) return MAGICPIG_UNSUPPORTED;   // (the kernels count its rows in 32 bits)
  // rows inside a page are addressed by 32-bit byte offsets
  if (key > ((int64_t)1 << 31) || row_bytes(p, key * p->page_size) >= ((int64_t)1 << 31)) return MAGICPIG_UNSUPPORTED;
  return MAGICPIG_OK;
}
int check_pools(const Params* p) {
  const int st = check_pool(p, p->k_stride_page, p->k_stride_key, p->k_stride_head);
  return st != MAGICPIG_OK ? st : check_pool(p, p->v_stride_page, p->v_stride_key, p->v_stride_head);
}
int check_rows(int64_t token, int64_t head) {
  if (token < 0 || head < 0) return MAGICPIG_INVALID_ARG;
  return (token | head) & 7 ? MAGICPIG_UNSUPPORTED : MAGICPIG_OK;
}

mp::PagedForm form_of(const Params* p, bool starts) {
  return mp::paged_form(p->batch, p->n_kv_heads, p->n_q_heads / p->n_kv_heads, p->dtype == MAGICPIG_FP32, p->max_tokens, starts ? most_new(p) : 1,
                        starts, (int64_t)p->max_pages * p->page_size, p->n_sink, p->n_local,
                        p->k_stride_head == mp::kHeadDim && p->v_stride_head == mp::kHeadDim ? (int)row_bytes(p, mp::kHeadDim) : 0, four(p));
}
// The workspace: counters of arrived partials (zero between calls), then what a call keeps for itself.
constexpr size_t kCounterBytes = MAGICPIG_PAGED_COUNTER_BYTES;
static_assert(kCounterBytes == mp::kPagedCounters * sizeof(unsigned), "");
size_t ws_attention(const mp::PagedForm& f) { return kCounterBytes + align256((size_t)f.slots * f.rows * mp::kPartialStride * sizeof(float)); }
size_t ws_plan(const Params* p) {
  return !mp::page_plan_needs_workspace(p->batch, p->max_tokens) ? 0 : kCounterBytes + align256((size_t)3 * (p->batch + 1) * sizeof(int));
}

int keep_parts_of(const Params* p) { return mp::keep_parts((int64_t)p->batch * p->n_kv_heads, (int64_t)p->max_pages * p->page_size); }
size_t ws_keep(const Params* p) {
  const int parts = keep_parts_of(p);
  return parts == 1 ? 0 : kCounterBytes + align256((size_t)p->batch * p->n_kv_heads * parts * mp::kKeepPartBytes);
}

// Attention over pools of any kind, behind check().
int attend(const Params* p, const void* q, const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale,
           const uint8_t* k_block, const uint8_t* v_block, const int32_t* block_table, const int32_t* lengths, const int32_t* token_start,
           void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int st;
  if ((st = check_pools(p)) != MAGICPIG_OK) return st;
  if ((st = check_rows(p->q_stride_token, p->q_stride_head)) != MAGICPIG_OK) return st;
  if (!token_start && p->max_tokens < p->batch) return MAGICPIG_INVALID_ARG;   // (row b of request b)
  if (!q || !k_pages || !v_pages || !out || (p->batch > 0 && (!block_table || !lengths))) return MAGICPIG_INVALID_ARG;
  if (p->kv_dtype != MAGICPIG_KV_FP8_E4M3 && (k_scale || v_scale)) return MAGICPIG_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(block_table, 4) ||
      !aligned(lengths, 4) || !aligned(token_start, 4) || !aligned16(out) || !aligned(lse, 4) || !aligned16(workspace))
    return MAGICPIG_INVALID_ARG;
  const mp::PagedForm f = form_of(p, token_start != nullptr);
  if (!mp::paged_grid_fits(f)) return MAGICPIG_UNSUPPORTED;
  const size_t need = ws_attention(f);
  if (!workspace || workspace_bytes < need) return MAGICPIG_WORKSPACE_TOO_SMALL;
  if (p->batch == 0) return MAGICPIG_OK;
  mp::PagedArgs a{};
  a.q = q; a.k = k_pages; a.v = v_pages; a.k_scale = k_scale; a.v_scale = v_scale;
  a.k_block = k_block; a.v_block = v_block;
  a.k_page_rows = (uint32_t)(p->k_stride_page / mp::kHeadDim); a.k_key_rows = (uint32_t)(p->k_stride_key / mp::kHeadDim);
  a.v_page_rows = (uint32_t)(p->v_stride_page / mp::kHeadDim); a.v_key_rows = (uint32_t)(p->v_stride_key / mp::kHeadDim);
  a.same_strides = p->k_stride_page == p->v_stride_page && p->k_stride_key == p->v_stride_key;
  a.table = block_table; a.lengths = lengths; a.token_start = token_start;
  a.out = out; a.lse = lse;
  a.arrived = reinterpret_cast<unsigned*>(workspace);
  a.partial = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + kCounterBytes);
  a.batch = p->batch; a.Hq = p->n_q_heads; a.Hkv = p->n_kv_heads; a.G = p->n_q_heads / p->n_kv_heads;
  a.page_shift = __builtin_ctz(p->page_size); a.max_pages = p->max_pages; a.max_new = token_start ? most_new(p) : 1;
  a.n_sink = p->n_sink; a.n_local = p->n_local;
  a.max_len = p->max_pages * p->page_size; a.max_tokens = (int)p->max_tokens; a.n_pages = (int)p->n_pages;
  a.tile_tokens = f.tile_tokens; a.head_blocks = f.head_blocks;
  a.scale_log2 = (p->scale == 0.f ? 0.08838834764831845f : p->scale) * kLog2e;
  a.per_piece = 1.0001f / (float)f.target;                  // (the margin keeps float32's rounding from making more pieces)
  a.target = f.target; a.min_tiles = f.min_tiles; a.slots = (int)f.slots;
  a.near_shift = f.near_shift; a.set_shift = f.set_shift; a.group_shift = f.group_shift;
  for (int i = 0; i <= f.set_shift; ++i) a.shares[i] = f.shares[i];
  a.k_page = p->k_stride_page; a.k_key = p->k_stride_key; a.k_head = p->k_stride_head;
  a.v_page = p->v_stride_page; a.v_key = p->v_stride_key; a.v_head = p->v_stride_head;
  a.q_t = p->q_stride_token; a.q_h = p->q_stride_head;
  const int element = four(p) ? mp::kFP4 : (p->kv_dtype == MAGICPIG_KV_FP8_E4M3 ? mp::kFP8 : (p->dtype == MAGICPIG_FP32 ? mp::kFP32 : mp::kBF16));
  return mp::hip_status(mp::launch_paged_attention(a, element, f, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // namespace

extern "C" {

size_t magicpig_paged_workspace_bytes(const Params* p) {
  if (check(p) != MAGICPIG_OK) return 0;
  size_t m = ws_plan(p);
  for (const bool starts : {false, true}) {
    const mp::PagedForm f = form_of(p, starts);
    const size_t a = mp::paged_grid_fits(f) ? ws_attention(f) : 0;   // (attention refuses the others)
    if (a > m) m = a;
  }
  const size_t keep = ws_keep(p);
  if (keep > m) m = keep;
  return m < 256 ? 256 : m;
}

int magicpig_page_plan(const Params* p, const int32_t* new_tokens, const int32_t* lengths, int32_t* block_table, int32_t* free_pages,
                       const int32_t* n_free, int32_t* lengths_out, int32_t* n_free_out, int32_t* token_start, int64_t* slots,
                       int32_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if (!free_pages || !n_free || !n_free_out || !token_start || !slots || !status) return MAGICPIG_INVALID_ARG;
  if (p->batch > 0 && (!new_tokens || !lengths || !block_table || !lengths_out)) return MAGICPIG_INVALID_ARG;
  if (!aligned(new_tokens, 4) || !aligned(lengths, 4) || !aligned(block_table, 4) || !aligned(free_pages, 4) || !aligned(n_free, 4) ||
      !aligned(lengths_out, 4) || !aligned(n_free_out, 4) || !aligned(token_start, 4) || !aligned(slots, 8) || !aligned(status, 4) ||
      !aligned16(workspace))
    return MAGICPIG_INVALID_ARG;
  const size_t need = ws_plan(p);
  if (need > 0 && (!workspace || workspace_bytes < need)) return MAGICPIG_WORKSPACE_TOO_SMALL;
  mp::PagePlanArgs a{};
  a.new_tokens = new_tokens; a.lengths = lengths; a.table = block_table; a.free_pages = free_pages; a.n_free = n_free;
  a.lengths_out = lengths_out; a.n_free_out = n_free_out; a.token_start = token_start; a.slots = slots; a.status = status;
  if (need > 0) a.scan = reinterpret_cast<int*>(reinterpret_cast<char*>(workspace) + kCounterBytes);
  a.batch = p->batch; a.page_shift = __builtin_ctz(p->page_size); a.max_pages = p->max_pages; a.max_new = p->max_new;
  a.n_pages = p->n_pages; a.max_tokens = p->max_tokens;
  return mp::hip_status(mp::launch_page_plan(a, reinterpret_cast<hipStream_t>(hip_stream)));
}

int magicpig_page_append(const Params* p, const void* k_new, const void* v_new, const int64_t* slots, const float* k_scale,
                         const float* v_scale, void* k_pages, void* v_pages, void* hip_stream) {
  int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if (four(p)) return MAGICPIG_UNSUPPORTED;
  if ((st = check_pools(p)) != MAGICPIG_OK) return st;
  if ((st = check_rows(p->k_new_stride_token, p->k_new_stride_head)) != MAGICPIG_OK) return st;
  if ((st = check_rows(p->v_new_stride_token, p->v_new_stride_head)) != MAGICPIG_OK) return st;
  if (!k_new || !v_new || !slots || !k_pages || !v_pages) return MAGICPIG_INVALID_ARG;
  if (p->kv_dtype != MAGICPIG_KV_FP8_E4M3 && (k_scale || v_scale)) return MAGICPIG_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned(slots, 8) || !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned16(k_pages) ||
      !aligned16(v_pages))
    return MAGICPIG_INVALID_ARG;
  mp::PageAppendArgs a{};
  a.k_new = k_new; a.v_new = v_new; a.slots = slots; a.k_scale = k_scale; a.v_scale = v_scale;
  a.k_pages = k_pages; a.v_pages = v_pages;
  a.heads = p->n_kv_heads; a.page_shift = __builtin_ctz(p->page_size);
  a.is_fp32 = p->dtype == MAGICPIG_FP32; a.kv_fp8 = p->kv_dtype == MAGICPIG_KV_FP8_E4M3;
  a.n_slots = p->n_pages * p->page_size; a.tokens = p->max_tokens;
  a.kn_t = p->k_new_stride_token; a.kn_h = p->k_new_stride_head; a.vn_t = p->v_new_stride_token; a.vn_h = p->v_new_stride_head;
  a.k_page = p->k_stride_page; a.k_key = p->k_stride_key; a.k_head = p->k_stride_head;
  a.v_page = p->v_stride_page; a.v_key = p->v_stride_key; a.v_head = p->v_stride_head;
  return mp::hip_status(mp::launch_page_append(a, reinterpret_cast<hipStream_t>(hip_stream)));
}

int magicpig_paged_attention(const Params* p, const void* q, const void* k_pages, const void* v_pages, const float* k_scale,
                             const float* v_scale, const int32_t* block_table, const int32_t* lengths, const int32_t* token_start, void* out,
                             float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if (four(p)) return MAGICPIG_UNSUPPORTED;
  return attend(p, q, k_pages, v_pages, k_scale, v_scale, nullptr, nullptr, block_table, lengths, token_start, out, lse, workspace,
                workspace_bytes, hip_stream);
}

int magicpig_paged_attention_mxfp(const Params* p, const void* q, const void* k_pages, const void* v_pages, const uint8_t* k_block_scales,
                                   const uint8_t* v_block_scales, const int32_t* block_table, const int32_t* lengths, const int32_t* token_start,
                                   void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if (!four(p)) return MAGICPIG_UNSUPPORTED;
  if (!k_block_scales || !v_block_scales || !aligned(k_block_scales, 4) || !aligned(v_block_scales, 4)) return MAGICPIG_INVALID_ARG;
  return attend(p, q, k_pages, v_pages, nullptr, nullptr, k_block_scales, v_block_scales, block_table, lengths, token_start, out, lse, workspace,
                workspace_bytes, hip_stream);
}

namespace {

// Rows to or from pools in four bits; the rows are written by a call that reads the pools.
int check_mxfp4(const Params* p, const void* k_rows, const void* v_rows, const int64_t* slots, const void* k_pages, const void* v_pages,
                const uint8_t* k_block, const uint8_t* v_block) {
  int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if (!four(p)) return MAGICPIG_UNSUPPORTED;
  if ((st = check_pools(p)) != MAGICPIG_OK) return st;
  if ((st = check_rows(p->k_new_stride_token, p->k_new_stride_head)) != MAGICPIG_OK) return st;
  if ((st = check_rows(p->v_new_stride_token, p->v_new_stride_head)) != MAGICPIG_OK) return st;
  if (!k_rows || !v_rows || !slots || !k_pages || !v_pages || !k_block || !v_block) return MAGICPIG_INVALID_ARG;
  if (!aligned16(k_rows) || !aligned16(v_rows) || !aligned(slots, 8) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned(k_block, 4) ||
      !aligned(v_block, 4))
    return MAGICPIG_INVALID_ARG;
  return MAGICPIG_OK;
}

mp::PageMxfp4Args mxfp4_args(const Params* p, const void* k_rows, const void* v_rows, const int64_t* slots, const void* k_pages,
                             const void* v_pages, const uint8_t* k_block, const uint8_t* v_block) {
  mp::PageMxfp4Args a{};
  a.k_rows = const_cast<void*>(k_rows); a.v_rows = const_cast<void*>(v_rows); a.slots = slots;
  a.k_pages = static_cast<uint8_t*>(const_cast<void*>(k_pages)); a.v_pages = static_cast<uint8_t*>(const_cast<void*>(v_pages));
  a.k_block = const_cast<uint8_t*>(k_block); a.v_block = const_cast<uint8_t*>(v_block);
  a.heads = p->n_kv_heads; a.page_shift = __builtin_ctz(p->page_size);
  a.n_slots = p->n_pages * p->page_size; a.tokens = p->max_tokens;
  a.kn_t = p->k_new_stride_token; a.kn_h = p->k_new_stride_head; a.vn_t = p->v_new_stride_token; a.vn_h = p->v_new_stride_head;
  a.k_page = p->k_stride_page; a.k_key = p->k_stride_key; a.k_head = p->k_stride_head;
  a.v_page = p->v_stride_page; a.v_key = p->v_stride_key; a.v_head = p->v_stride_head;
  return a;
}

}  // namespace

int magicpig_page_append_mxfp(const Params* p, const void* k_new, const void* v_new, const int64_t* slots, void* k_pages, void* v_pages,
                               uint8_t* k_block_scales, uint8_t* v_block_scales, void* hip_stream) {
  const int st = check_mxfp4(p, k_new, v_new, slots, k_pages, v_pages, k_block_scales, v_block_scales);
  if (st != MAGICPIG_OK) return st;
  return mp::hip_status(mp::launch_page_append_mxfp4(mxfp4_args(p, k_new, v_new, slots, k_pages, v_pages, k_block_scales, v_block_scales),
                                                     reinterpret_cast<hipStream_t>(hip_stream)));
}

int magicpig_page_read_mxfp(const Params* p, const void* k_pages, const void* v_pages, const uint8_t* k_block_scales,
                             const uint8_t* v_block_scales, const int64_t* slots, void* k_out, void* v_out, void* hip_stream) {
  const int st = check_mxfp4(p, k_out, v_out, slots, k_pages, v_pages, k_block_scales, v_block_scales);
  if (st != MAGICPIG_OK) return st;
  return mp::hip_status(mp::launch_page_read_mxfp4(mxfp4_args(p, k_out, v_out, slots, k_pages, v_pages, k_block_scales, v_block_scales),
                                                   reinterpret_cast<hipStream_t>(hip_stream)));
}

namespace {

mp::WeightsForm weights_form_of(const Params* p, bool starts) {
  return mp::weights_form(p->batch, p->n_kv_heads, p->n_q_heads / p->n_kv_heads, p->dtype == MAGICPIG_FP32,
                          four(p) ? 4 : (p->kv_dtype == MAGICPIG_KV_FP8_E4M3 ? 8 : 16), starts ? most_new(p) : 1, (int64_t)p->max_pages * p->page_size);
}

}  // namespace

int magicpig_page_weights(const Params* p, const void* q, const void* k_pages, const float* k_scale, const uint8_t* k_block_scales,
                          const int32_t* block_table, const int32_t* lengths, const int32_t* token_start, const float* lse,
                          const int32_t* counted, float* weights, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if ((st = check_pool(p, p->k_stride_page, p->k_stride_key, p->k_stride_head)) != MAGICPIG_OK) return st;
  if ((st = check_rows(p->q_stride_token, p->q_stride_head)) != MAGICPIG_OK) return st;
  if (!token_start && p->max_tokens < p->batch) return MAGICPIG_INVALID_ARG;
  if (!q || !k_pages || !lse || !weights || (p->batch > 0 && (!block_table || !lengths))) return MAGICPIG_INVALID_ARG;
  if (k_scale && p->kv_dtype != MAGICPIG_KV_FP8_E4M3) return MAGICPIG_INVALID_ARG;
  if (four(p) ? !k_block_scales : k_block_scales != nullptr) return MAGICPIG_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned(k_scale, 4) || !aligned(k_block_scales, 4) || !aligned(block_table, 4) ||
      !aligned(lengths, 4) || !aligned(token_start, 4) || !aligned(lse, 4) || !aligned(counted, 4) || !aligned(weights, 4) || !aligned16(workspace))
    return MAGICPIG_INVALID_ARG;
  const mp::WeightsForm f = weights_form_of(p, token_start != nullptr);
  if (!mp::weights_fit(f)) return MAGICPIG_UNSUPPORTED;
  if (p->q_stride_token > (1 << 22) || p->q_stride_head > (1 << 22)) return MAGICPIG_UNSUPPORTED;   // (a tile's rows lie within 2^31 bytes)
  (void)workspace_bytes;
  if (p->batch == 0) return MAGICPIG_OK;
  mp::PageWeightsArgs a{};
  a.paged.q = q; a.paged.k = k_pages; a.paged.k_scale = k_scale; a.paged.k_block = k_block_scales;
  a.paged.table = block_table; a.paged.lengths = lengths; a.paged.token_start = token_start;
  a.paged.batch = p->batch; a.paged.Hq = p->n_q_heads; a.paged.Hkv = p->n_kv_heads; a.paged.G = p->n_q_heads / p->n_kv_heads;
  a.paged.page_shift = __builtin_ctz(p->page_size); a.paged.max_pages = p->max_pages; a.paged.max_new = token_start ? most_new(p) : 1;
  a.paged.n_sink = p->n_sink; a.paged.n_local = p->n_local;
  a.paged.max_len = p->max_pages * p->page_size; a.paged.max_tokens = (int)p->max_tokens; a.paged.n_pages = (int)p->n_pages;
  a.paged.scale_log2 = (p->scale == 0.f ? 0.08838834764831845f : p->scale) * kLog2e;
  a.paged.k_page = p->k_stride_page; a.paged.k_key = p->k_stride_key; a.paged.k_head = p->k_stride_head;
  a.paged.q_t = p->q_stride_token; a.paged.q_h = p->q_stride_head;
  a.lse = lse; a.counted = counted; a.weights = weights; a.heads = f.heads;
  const int element = four(p) ? mp::kFP4 : (p->kv_dtype == MAGICPIG_KV_FP8_E4M3 ? mp::kFP8 : (p->dtype == MAGICPIG_FP32 ? mp::kFP32 : mp::kBF16));
  return mp::hip_status(mp::launch_page_weights(a, element, f, reinterpret_cast<hipStream_t>(hip_stream)));
}

int magicpig_page_keep(const Params* p, const float* weights, const int32_t* block_table, const int32_t* lengths, const int32_t* budgets,
                       int32_t n_first, int32_t n_last, int32_t max_keep, int32_t* kept, int32_t* lengths_out, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  const int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if (n_first < 0 || n_last < 0 || max_keep < 1) return MAGICPIG_INVALID_ARG;
  if (max_keep > (1 << 30)) return MAGICPIG_UNSUPPORTED;   // (no request has more keys)
  if ((int64_t)p->batch * p->n_kv_heads * 1024 >= (int64_t)1 << 32) return MAGICPIG_UNSUPPORTED;   // (threads of a grid)
  if (p->batch > 0 && (!weights || !block_table || !lengths || !budgets || !kept || !lengths_out)) return MAGICPIG_INVALID_ARG;
  if (!aligned16(weights) || !aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(budgets, 4) || !aligned(kept, 4) ||
      !aligned(lengths_out, 4) || !aligned16(workspace))
    return MAGICPIG_INVALID_ARG;
  const size_t need = ws_keep(p);
  if (need > 0 && (!workspace || workspace_bytes < need)) return MAGICPIG_WORKSPACE_TOO_SMALL;
  if (p->batch == 0) return MAGICPIG_OK;
  mp::PageKeepArgs a{};
  a.weights = weights; a.table = block_table; a.lengths = lengths; a.budgets = budgets; a.kept = kept; a.lengths_out = lengths_out;
  a.batch = p->batch; a.heads = p->n_kv_heads; a.page_shift = __builtin_ctz(p->page_size); a.max_pages = p->max_pages;
  a.max_len = p->max_pages * p->page_size; a.n_pages = (int)p->n_pages; a.n_first = n_first; a.n_last = n_last; a.max_keep = max_keep;
  a.parts = keep_parts_of(p);
  if (need > 0) a.workspace = reinterpret_cast<char*>(workspace) + kCounterBytes;
  return mp::hip_status(mp::launch_page_keep(a, (int64_t)p->batch * p->n_kv_heads, reinterpret_cast<hipStream_t>(hip_stream)));
}

int magicpig_page_evict(const Params* p, const int32_t* kept, int32_t max_keep, const int32_t* lengths, const int32_t* lengths_kept,
                        const int32_t* block_table, int32_t* free_pages, const int32_t* n_free, void* k_pages, void* v_pages,
                        uint8_t* k_block_scales, uint8_t* v_block_scales, float* weights, int32_t* n_free_out, int32_t* status,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  int st = check(p);
  if (st != MAGICPIG_OK) return st;
  if ((st = check_pools(p)) != MAGICPIG_OK) return st;
  if (kept && max_keep < 1) return MAGICPIG_INVALID_ARG;
  if (kept && max_keep > (1 << 30)) return MAGICPIG_UNSUPPORTED;
  if (!free_pages || !n_free || !n_free_out || !status || !k_pages || !v_pages) return MAGICPIG_INVALID_ARG;
  if (p->batch > 0 && (!lengths || !lengths_kept || !block_table)) return MAGICPIG_INVALID_ARG;
  if (four(p) ? !k_block_scales || !v_block_scales : k_block_scales || v_block_scales) return MAGICPIG_INVALID_ARG;
  if (!aligned(kept, 4) || !aligned(lengths, 4) || !aligned(lengths_kept, 4) || !aligned(block_table, 4) || !aligned(free_pages, 4) ||
      !aligned(n_free, 4) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned(k_block_scales, 4) || !aligned(v_block_scales, 4) ||
      !aligned(weights, 4) || !aligned(n_free_out, 4) || !aligned(status, 4) || !aligned16(workspace))
    return MAGICPIG_INVALID_ARG;
  (void)workspace_bytes;
  mp::PageEvictArgs a{};
  a.kept = kept; a.lengths = lengths; a.stay = lengths_kept; a.table = block_table; a.free_pages = free_pages; a.n_free = n_free;
  a.n_free_out = n_free_out; a.status = status;
  a.batch = p->batch; a.heads = p->n_kv_heads; a.page_shift = __builtin_ctz(p->page_size); a.max_pages = p->max_pages;
  a.max_len = p->max_pages * p->page_size; a.max_keep = max_keep; a.n_pages = p->n_pages;
  const int row = (int)row_bytes(p, mp::kHeadDim), slice = mp::evict_slice(row, (int64_t)p->batch * p->n_kv_heads);
  auto array = [](void* at, int64_t page, int64_t key, int64_t head, int slice, int slices) {
    return mp::PagedArray{static_cast<char*>(at), page, key, head, slice, slices};
  };
  a.arrays[0] = array(k_pages, row_bytes(p, p->k_stride_page), row_bytes(p, p->k_stride_key), row_bytes(p, p->k_stride_head), slice, row / slice);
  a.arrays[1] = array(v_pages, row_bytes(p, p->v_stride_page), row_bytes(p, p->v_stride_key), row_bytes(p, p->v_stride_head), slice, row / slice);
  if (weights) a.arrays[2] = array(weights, (int64_t)p->n_kv_heads * p->page_size * 4, 4, (int64_t)p->page_size * 4, 4, 1);
  if (four(p)) {
    a.arrays[3] = array(k_block_scales, p->k_stride_page / 32, p->k_stride_key / 32, p->k_stride_head / 32, 4, 1);
    a.arrays[4] = array(v_block_scales, p->v_stride_page / 32, p->v_stride_key / 32, p->v_stride_head / 32, 4, 1);
  }
  return mp::hip_status(mp::launch_page_evict(a, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
