// Entry points of the sampling phase: argument checks on the host, then the launches on the caller's stream.  Nothing here
// allocates device memory or synchronises; a plan is host data.
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <new>

#include "paged.h"

namespace {

bool misaligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

int element_size(int32_t dtype) { return dtype == PA_BF16 ? 2 : 4; }

int check_rope(const rope_axes_desc_t* d) {
  if (!d) return PA_ERR_NULL;
  if (d->head_dim < 2 || d->head_dim > 2 * PA_ROPE_MAX_PAIRS) return PA_ERR_SHAPE;
  if (d->rotary_dim < 2 || d->rotary_dim > d->head_dim || d->rotary_dim % 2) return PA_ERR_SHAPE;
  if (d->num_axes < 1 || d->num_axes > PA_ROPE_MAX_AXES) return PA_ERR_SHAPE;
  if (d->layout != PA_ROPE_HALVES && d->layout != PA_ROPE_PAIRS) return PA_ERR_UNSUPPORTED;
  for (int i = 0; i < d->rotary_dim / 2; ++i)
    if (d->pair_axis[i] >= d->num_axes) return PA_ERR_SHAPE;
  return PA_OK;
}

// `tokens` rows of `heads` heads, `stride` elements apart
int check_rows(const void* p, int64_t stride, int32_t heads, int32_t D, int32_t dtype) {
  if (!p) return PA_ERR_NULL;
  if (stride < (int64_t)heads * D || stride > ((int64_t)1 << 40)) return PA_ERR_SHAPE;
  if (misaligned(p, (uintptr_t)element_size(dtype))) return PA_ERR_ALIGN;
  return PA_OK;
}

int rope_call(const rope_axes_desc_t* desc, int32_t dtype, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
              int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads, const int32_t* positions, const float* inv_freq,
              void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* hip_stream, float sign) {
  int st = check_rope(desc);
  if (st != PA_OK) return st;
  if (dtype != PA_F32 && dtype != PA_BF16) return PA_ERR_UNSUPPORTED;
  if (num_tokens < 0 || num_tokens > ((int64_t)1 << 31) - 1 || num_q_heads < 1 || num_q_heads > 65536 || num_k_heads < 0 ||
      num_k_heads > 65536)
    return PA_ERR_SHAPE;
  if (num_tokens == 0) return PA_OK;
  if (!positions || !inv_freq) return PA_ERR_NULL;
  if ((st = check_rows(q, q_stride, num_q_heads, desc->head_dim, dtype)) != PA_OK) return st;
  if ((st = check_rows(q_out, q_out_stride, num_q_heads, desc->head_dim, dtype)) != PA_OK) return st;
  if (num_k_heads > 0) {
    if ((st = check_rows(k, k_stride, num_k_heads, desc->head_dim, dtype)) != PA_OK) return st;
    if ((st = check_rows(k_out, k_out_stride, num_k_heads, desc->head_dim, dtype)) != PA_OK) return st;
  }
  if (misaligned(positions, 4) || misaligned(inv_freq, 4)) return PA_ERR_ALIGN;
  pa::RopeArgs a{};
  a.rope = *desc;
  a.dtype = dtype;
  a.Hq = num_q_heads;
  a.Hk = num_k_heads;
  a.sign = sign;
  a.T = num_tokens;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.q_out_stride = q_out_stride;
  a.k_out_stride = k_out_stride;
  a.positions = positions;
  a.inv_freq = inv_freq;
  return pa::launch_rope(a, hip_stream) == 0 ? PA_OK : PA_ERR_HIP;
}

// What every call on a plan checks; `empty` is set when there is nothing to do.
int check_call(const paged_attn_plan_t* plan, const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new,
               int32_t num_seqs, int64_t num_tokens, bool* empty) {
  if (!plan) return PA_ERR_NULL;
  const paged_attn_desc_t& d = plan->desc;
  if (num_seqs < 0 || num_seqs > d.max_seqs || num_tokens < 0 || num_tokens > d.max_tokens) return PA_ERR_SHAPE;
  *empty = num_seqs == 0 || num_tokens == 0;
  if (*empty) return PA_OK;
  if (!page_table || !seq_lens || !cu_new) return PA_ERR_NULL;
  if (misaligned(page_table, 4) || misaligned(seq_lens, 4) || misaligned(cu_new, 4)) return PA_ERR_ALIGN;
  return PA_OK;
}

// Host-only plans and other devices: after all other checks, so that those can be tested without a device.
int check_device(const paged_attn_desc_t& d) {
  if (d.device < 0) return PA_ERR_UNSUPPORTED;
  int cur = -1;
  return hipGetDevice(&cur) == hipSuccess && cur == d.device ? PA_OK : PA_ERR_HIP;  // the plan's device must be current
}

int append_call(const paged_attn_plan_t* plan, const rope_axes_desc_t* rope, const void* q, int64_t q_stride, const void* k,
                int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions, const float* inv_freq,
                void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache, const int32_t* page_table,
                const int32_t* seq_lens, const int32_t* cu_new, int32_t num_seqs, int64_t num_tokens, void* hip_stream) {
  bool empty = false;
  int st = check_call(plan, page_table, seq_lens, cu_new, num_seqs, num_tokens, &empty);
  if (st != PA_OK || empty) return st;
  const paged_attn_desc_t& d = plan->desc;
  if ((st = check_rows(k, k_stride, d.num_kv_heads, d.head_dim, d.dtype)) != PA_OK) return st;
  if ((st = check_rows(v, v_stride, d.num_kv_heads, d.head_dim, d.dtype)) != PA_OK) return st;
  if (!k_cache || !v_cache) return PA_ERR_NULL;
  if (misaligned(k_cache, 16) || misaligned(v_cache, 16)) return PA_ERR_ALIGN;
  pa::RopeArgs a{};
  if (rope) {
    if (rope->head_dim != d.head_dim) return PA_ERR_SHAPE;
    if (!positions || !inv_freq || !q != !q_out) return PA_ERR_NULL;
    if (misaligned(positions, 4) || misaligned(inv_freq, 4)) return PA_ERR_ALIGN;
    a.rope = *rope;
    if (q) {
      if ((st = check_rows(q, q_stride, d.num_q_heads, d.head_dim, d.dtype)) != PA_OK) return st;
      if ((st = check_rows(q_out, q_out_stride, d.num_q_heads, d.head_dim, d.dtype)) != PA_OK) return st;
      a.Hq = d.num_q_heads;
    }
  } else {
    a.rope.head_dim = d.head_dim;
    a.rope.layout = PA_ROPE_HALVES;
  }
  if ((st = check_device(d)) != PA_OK) return st;
  a.dtype = d.dtype;
  a.Hk = a.Hv = d.num_kv_heads;
  a.sign = 1.f;
  a.T = num_tokens;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.page_table = page_table;
  a.seq_lens = seq_lens;
  a.cu_new = cu_new;
  a.B = num_seqs;
  a.table_width = d.max_pages_per_seq;
  a.page_shift = plan->page_shift;
  a.num_pages = d.num_pages;
  return pa::launch_append(a, hip_stream) == 0 ? PA_OK : PA_ERR_HIP;
}

// Rows of a block for an average of `rows` rows a sequence (with shared keys: rows in all, which their blocks hold together).
int32_t blocks16_for(int64_t rows, int32_t dtype) { return rows <= 16 ? 1 : rows <= 32 || dtype == PA_F32 ? 2 : 4; }

// A bf16 call of at most this many rows a sequence, on average, is one of few rows.  Measured with either kernel for all calls, few rows and chunks (16
// sequences of 2,000 ... 6,000 keys, 28 + 4 heads of 128): 14 rows 34 and 44 us, 56 rows 44 and 47, 63 rows 47 and 48, 70 rows 53 and 50,
// 126 rows 59 and 55, 252 rows 93 and 76; 32 sequences of 4 + 4 heads: 64 rows 64 and 66, 80 rows 92 and 71; 24 of 14 + 2 heads of 64: 63 rows
// 33 and 37, 126 rows 39 and 40, 252 rows 54 and 50.  The average says little where single tokens run beside one long chunk: 127 of them and
// a chunk of 1,000 (61.6 rows) take 245 us, 165 in the other kernel, 64 and 512 (62 rows) 294 and 249.
constexpr int64_t FEW_ROWS = 64;
// Up to this many rows a sequence, on average, shared keys are a segment of their own.  They save passes over these keys while the blocks
// of one sequence's rows are not nearly full, and cost a piece more of every row.  With and without, 4, 8, 16 and 64 sequences over 32,768 shared keys, 28 + 4
// heads of 128: 7 rows 31 and 53, 34 and 91, 49 and 165, 126 and 512 us; 35 rows 52 and 72, 80 and 104, 135 and 179, 418 and 583; 56 rows 64 and 80,
// 112 and 109, 183 and 183, 691 and 582; 63 rows 66 and 83, 132 and 110, 239 and 184, 808 and 584.  fp32 (8 + 2 heads, 32 sequences over 8,192):
// 48 rows 175 and 199, 64 rows 225 and 202.
constexpr int64_t SHARED_ROWS = 56;

// What starting and ending a block costs, in keys, and the least share (that cost included) worth a workgroup and a merge.  Measured over
// 32 ... 480 keys: one token over 1,100 keys 16.4 us with 64 (and 256), 14.8 with 240 (320); eight rollouts over a shared video 36.7
// and 33.6; fp32 chunks 74 with 64, 65 with 160, 67.5 with 240; chunks of 1 ... 301 tokens (24 sequences, heads of 64) 157 with 128
// (512), 149 with 384 (768); a single chunk of 2,048 tokens does not mind.
struct Costs {
  int32_t start_keys, min_share;
};
constexpr Costs FEW_ROWS_COSTS[2] = {{160, 256}, {240, 320}};  // fp32, bf16
constexpr Costs CHUNK_COSTS = {384, 768};

// bf16 calls of more rows a sequence than a block of few rows holds run in blocks of PAGED_CHUNK_ROWS
bool is_chunk(int64_t rows, int64_t num_seqs, int32_t dtype) { return dtype == PA_BF16 && rows > FEW_ROWS * num_seqs; }

pa::PagedArgs arrange(const paged_attn_plan_t& plan, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache,
                      const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new, int32_t num_seqs, int32_t num_tokens,
                      const int32_t* shared_len, void* out, float* lse_out, char* ws) {
  const paged_attn_desc_t& d = plan.desc;
  pa::PagedArgs a{};
  a.q = q;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.out = out;
  a.lse = lse_out;
  a.page_table = page_table;
  a.seq_lens = seq_lens;
  a.cu_new = cu_new;
  a.q_stride = q_stride;
  a.num_pages = d.num_pages;
  a.dtype = d.dtype;
  a.D = d.head_dim;
  a.Hq = d.num_q_heads;
  a.table_width = d.max_pages_per_seq;
  a.page_shift = plan.page_shift;
  a.scale = d.softmax_scale;
  const int64_t rows = (int64_t)num_tokens * plan.group;
  a.shared_len = rows <= SHARED_ROWS * num_seqs ? shared_len : nullptr;
  a.blocks16 = blocks16_for(a.shared_len ? rows : (rows + num_seqs - 1) / num_seqs, d.dtype);
  a.groups = plan.num_cu;
  a.xcd_shift = plan.xcd_shift;
  pa::PagedShape& s = a.shape;
  s.B = num_seqs;
  s.T = num_tokens;
  s.Hkv = d.num_kv_heads;
  s.group = plan.group;
  const bool chunk = is_chunk(rows, num_seqs, d.dtype);
  s.block_rows = chunk ? pa::PAGED_CHUNK_ROWS : 16 * a.blocks16;
  s.tile_shift = chunk ? pa::PAGED_CHUNK_TILE_SHIFT : pa::paged_rows_tile_shift(d.dtype, d.head_dim);
  // Single tokens beside chunks, whose wavefronts are half idle: 31 tokens and a chunk of 2,000 (28 + 4 heads of 128) 342 us at full cost,
  // 310 at half, 468 at a quarter; 95 and 3,000 (14 + 2 heads of 64) 227, 195 and 287.
  s.half_rows = chunk ? pa::PAGED_CHUNK_ROWS / 2 : 0;
  s.causal_cuts = chunk;
  s.inv_group = 1.0f / (float)s.group;
  s.capacity = d.max_pages_per_seq << plan.page_shift;
  const Costs costs = chunk ? CHUNK_COSTS : FEW_ROWS_COSTS[d.dtype == PA_BF16];
  // No lengths of such a call can cost more than this many keys; the unit keeps that below 2^30 units.
  const double most = ((double)rows / s.block_rows + 2.0 * (num_seqs + 1)) * s.Hkv * ((double)s.capacity + num_tokens + costs.start_keys + 64);
  s.unit_shift = 4;
  while (most / (double)((int64_t)1 << s.unit_shift) > (double)(1 << 29)) ++s.unit_shift;
  s.start_cost = (costs.start_keys >> s.unit_shift) + 1;
  s.min_share = (costs.min_share >> s.unit_shift) + 1;
  s.growth = (s.block_rows << pa::GROWTH_SHIFT) / s.group;
  s.per_group = (1.0f + 1.0f / (1 << 20)) / (float)a.groups;
  if (!ws) return a;  // the schedule alone
  a.line = reinterpret_cast<pa::PagedLine*>(ws);
  a.seg_start = reinterpret_cast<int32_t*>(ws + plan.off_seg_start);
  a.cuts = reinterpret_cast<pa::PagedCut*>(ws + plan.off_cuts);
  a.slot_lse = reinterpret_cast<float*>(ws + plan.off_slot_lse);
  a.slots = reinterpret_cast<float*>(ws + plan.off_slots);
  a.rows_lse = reinterpret_cast<float*>(ws + plan.off_rows_lse);
  a.rows = reinterpret_cast<float*>(ws + plan.off_rows);
  return a;
}

}  // namespace

extern "C" {

int rope_axes_forward(const rope_axes_desc_t* desc, int32_t dtype, const void* q, int64_t q_stride, const void* k,
                      int64_t k_stride, int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                      const int32_t* positions, const float* inv_freq, void* q_out, int64_t q_out_stride, void* k_out,
                      int64_t k_out_stride, void* hip_stream) {
  return rope_call(desc, dtype, q, q_stride, k, k_stride, num_tokens, num_q_heads, num_k_heads, positions, inv_freq, q_out,
                   q_out_stride, k_out, k_out_stride, hip_stream, 1.f);
}

int rope_axes_backward(const rope_axes_desc_t* desc, int32_t dtype, const void* q, int64_t q_stride, const void* k,
                       int64_t k_stride, int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads,
                       const int32_t* positions, const float* inv_freq, void* q_out, int64_t q_out_stride, void* k_out,
                       int64_t k_out_stride, void* hip_stream) {
  return rope_call(desc, dtype, q, q_stride, k, k_stride, num_tokens, num_q_heads, num_k_heads, positions, inv_freq, q_out,
                   q_out_stride, k_out, k_out_stride, hip_stream, -1.f);
}

int paged_attn_plan(const paged_attn_desc_t* desc, paged_attn_plan_t** plan_out, size_t* workspace_bytes_out) {
  if (plan_out) *plan_out = nullptr;
  if (!desc || !plan_out || !workspace_bytes_out) return PA_ERR_NULL;
  const paged_attn_desc_t& d = *desc;
  if (d.num_q_heads < 1 || d.num_kv_heads < 1 || d.num_q_heads % d.num_kv_heads || d.num_q_heads > 4096) return PA_ERR_SHAPE;
  if (d.num_pages < 1 || d.num_pages > ((int64_t)1 << 31) - 1) return PA_ERR_SHAPE;
  if (d.max_seqs < 1 || d.max_seqs > 65536 || d.max_tokens < 1 || d.max_tokens > (1 << 24)) return PA_ERR_SHAPE;
  if (d.max_tokens * d.num_q_heads > ((int64_t)1 << 31) - 1) return PA_ERR_SHAPE;  // rows are numbered in 32 bits
  if (!(d.softmax_scale > 0.0f) || !std::isfinite(d.softmax_scale) || d.device < -1) return PA_ERR_SHAPE;
  if (d.max_pages_per_seq < 1 || d.page_size < 1) return PA_ERR_SHAPE;
  if (d.head_dim != 64 && d.head_dim != 128) return PA_ERR_UNSUPPORTED;
  if (d.dtype != PA_F32 && d.dtype != PA_BF16) return PA_ERR_UNSUPPORTED;
  if (d.page_size < 16 || d.page_size > 1024 || (d.page_size & (d.page_size - 1))) return PA_ERR_UNSUPPORTED;
  if ((int64_t)d.max_pages_per_seq * d.page_size > ((int64_t)1 << 30)) return PA_ERR_SHAPE;
  paged_attn_plan_t* p = new (std::nothrow) paged_attn_plan_t;
  if (!p) return PA_ERR_ALLOC;
  p->desc = d;
  while ((1 << p->page_shift) < d.page_size) ++p->page_shift;
  p->group = d.num_q_heads / d.num_kv_heads;
  if (d.device >= 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, d.device) != hipSuccess || n < 1) {
      (void)hipGetLastError();
      delete p;
      return PA_ERR_HIP;
    }
    p->num_cu = n;
    p->xcd_shift = n == 256 ? 3 : 0;  // the layout that shares are spread over XCDs for
  }
  // What the shares leave of blocks that they cut, and, where shared keys are a segment of their own, partials of all rows.
  const int64_t block_rows = is_chunk(d.max_tokens * p->group, 1, d.dtype) ? pa::PAGED_CHUNK_ROWS : 64, slots = 2 * (int64_t)p->num_cu * block_rows;
  const int64_t most = SHARED_ROWS * d.max_seqs / p->group, tokens = most < d.max_tokens ? most : d.max_tokens;
  size_t at = 256;
  auto take = [&](size_t bytes) {
    const size_t off = at;
    at += (bytes + 255) / 256 * 256;
    return off;
  };
  p->off_seg_start = take(((size_t)d.max_seqs + 2) * sizeof(int32_t));
  p->off_cuts = take((size_t)p->num_cu * sizeof(pa::PagedCut));
  p->off_slot_lse = take((size_t)slots * sizeof(float));
  p->off_slots = take((size_t)slots * d.head_dim * sizeof(float));
  p->off_rows_lse = take((size_t)tokens * d.num_q_heads * 2 * sizeof(float));
  p->off_rows = take((size_t)tokens * d.num_q_heads * 2 * d.head_dim * sizeof(float));
  p->ws_bytes = at;
  *plan_out = p;
  *workspace_bytes_out = p->ws_bytes;
  return PA_OK;
}

void paged_attn_destroy(paged_attn_plan_t* plan) { delete plan; }

int paged_kv_append(const paged_attn_plan_t* plan, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                    void* k_cache, void* v_cache, const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new,
                    int32_t num_seqs, int64_t num_tokens, void* hip_stream) {
  return append_call(plan, nullptr, nullptr, 0, k, k_stride, v, v_stride, nullptr, nullptr, nullptr, 0, k_cache, v_cache,
                     page_table, seq_lens, cu_new, num_seqs, num_tokens, hip_stream);
}

int paged_kv_append_rope(const paged_attn_plan_t* plan, const rope_axes_desc_t* rope, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                         const float* inv_freq, void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache,
                         const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new, int32_t num_seqs,
                         int64_t num_tokens, void* hip_stream) {
  const int st = check_rope(rope);
  if (st != PA_OK) return st;
  return append_call(plan, rope, q, q_stride, k, k_stride, v, v_stride, positions, inv_freq, q_out, q_out_stride, k_cache,
                     v_cache, page_table, seq_lens, cu_new, num_seqs, num_tokens, hip_stream);
}

int paged_attn_forward(const paged_attn_plan_t* plan, const void* q, int64_t q_stride, const void* k_cache,
                       const void* v_cache, const int32_t* page_table, const int32_t* seq_lens, const int32_t* cu_new,
                       int32_t num_seqs, int64_t num_tokens, const int32_t* shared_len, void* out, float* lse_out,
                       void* workspace, size_t workspace_bytes, void* hip_stream) {
  bool empty = false;
  int st = check_call(plan, page_table, seq_lens, cu_new, num_seqs, num_tokens, &empty);
  if (st != PA_OK || empty) return st;
  const paged_attn_desc_t& d = plan->desc;
  if ((st = check_rows(q, q_stride, d.num_q_heads, d.head_dim, d.dtype)) != PA_OK) return st;
  if (!k_cache || !v_cache || !out || !workspace) return PA_ERR_NULL;
  if (misaligned(q, 16) || q_stride * element_size(d.dtype) % 16 || misaligned(k_cache, 16) || misaligned(v_cache, 16) ||
      misaligned(out, 16) || misaligned(workspace, 16) || misaligned(lse_out, 4) || misaligned(shared_len, 4))
    return PA_ERR_ALIGN;
  if (workspace_bytes < plan->ws_bytes) return PA_ERR_WORKSPACE;
  if ((st = check_device(d)) != PA_OK) return st;
  const pa::PagedArgs a = arrange(*plan, q, q_stride, k_cache, v_cache, page_table, seq_lens, cu_new, num_seqs, (int32_t)num_tokens,
                                  shared_len, out, lse_out, static_cast<char*>(workspace));
  const bool chunk = is_chunk(num_tokens * plan->group, num_seqs, d.dtype);
  if ((chunk ? pa::launch_paged_chunk(a, hip_stream) : pa::launch_paged_rows(a, hip_stream)) != 0) return PA_ERR_HIP;
  return pa::launch_paged_merge(a, hip_stream) == 0 ? PA_OK : PA_ERR_HIP;
}

int paged_attn_schedule_shape(const paged_attn_plan_t* plan, int32_t num_seqs, int64_t num_tokens, int32_t with_shared, int32_t* groups,
                              int32_t* block_rows, int32_t* tile_keys) {
  if (!plan || !groups || !block_rows || !tile_keys) return PA_ERR_NULL;
  if (num_seqs < 1 || num_seqs > plan->desc.max_seqs || num_tokens < 1 || num_tokens > plan->desc.max_tokens) return PA_ERR_SHAPE;
  const int32_t given = 0;
  const pa::PagedArgs a = arrange(*plan, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr, num_seqs, (int32_t)num_tokens,
                                  with_shared ? &given : nullptr, nullptr, nullptr, nullptr);
  *groups = a.groups;
  *block_rows = a.shape.block_rows;
  *tile_keys = 1 << a.shape.tile_shift;
  return PA_OK;
}

int64_t paged_attn_schedule(const paged_attn_plan_t* plan, const int32_t* seq_lens, const int32_t* cu_new, int32_t num_seqs,
                            int64_t num_tokens, int32_t shared_len, int32_t* pieces_out, int64_t max_pieces) {
  if (!plan || !seq_lens || !cu_new || (!pieces_out && max_pieces > 0)) return -PA_ERR_NULL;
  if (num_seqs < 1 || num_seqs > plan->desc.max_seqs || num_tokens < 1 || num_tokens > plan->desc.max_tokens) return -PA_ERR_SHAPE;
  const pa::PagedArgs a = arrange(*plan, nullptr, 0, nullptr, nullptr, nullptr, seq_lens, cu_new, num_seqs, (int32_t)num_tokens,
                                  shared_len >= 0 ? &shared_len : nullptr, nullptr, nullptr, nullptr);
  pa::PagedShape s = a.shape;
  const bool with = a.shared_len != nullptr;
  s.shared = with ? pa::whole_pages(s, shared_len, plan->page_shift) : 0;
  auto segment = [&](int i) {
    return with && i == 0 ? pa::shared_segment(s, cu_new[num_seqs])
                          : pa::own_segment(s, cu_new[i - with], cu_new[i - with + 1], seq_lens[i - with]);
  };
  int64_t count = 0;
  int32_t total = 0;
  for (int i = 0; i < num_seqs + with; ++i) {
    const int32_t cost = segment(i).cost;
    if (cost < 0) return 0;
    total += s.Hkv * cost;
  }
  const int32_t share = pa::share_of(s, total), active = pa::active_of(total, share);
  for (int32_t w = 0; w < active; ++w) {
    int32_t x = w * share, start = 0, i = 0;
    const int32_t end = x + share < total ? x + share : total;
    while (x < end) {
      const pa::Segment g = segment(i);
      if (start + s.Hkv * g.cost <= x) {
        start += s.Hkv * g.cost;
        ++i;
        continue;
      }
      const bool shared = with && i == 0;
      const int32_t head = pa::div_small(x - start, g.cost), head_start = start + head * g.cost, block = pa::block_at(s, g, x - head_start);
      const pa::Block b = pa::make_block(s, g, head_start, block);
      const pa::Piece p = pa::make_piece(s, g, shared, b, x, end);
      if (count < max_pieces) {
        const int32_t k1 = g.key0 + (p.tile1 << s.tile_shift);
        const int32_t row[8] = {w, shared ? -1 : i - (int)with, head, block * s.block_rows, b.rows, g.key0 + (p.tile0 << s.tile_shift),
                                k1 < p.key_end ? k1 : p.key_end, p.whole};
        for (int e = 0; e < 8; ++e) pieces_out[count * 8 + e] = row[e];
      }
      ++count;
      x = end < b.c1 ? end : b.c1;
    }
  }
  return count;
}

}  // extern "C"
