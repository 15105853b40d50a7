// Internal declarations of the sampling phase: rotary positions, paged cache and attention over pages.
#pragma once

#include <cstddef>
#include <cstdint>

#include "paged_attn.h"

namespace pa {

// What the rotation and the append kernel read and write.  Heads are numbered q first, then k, then v.
struct RopeArgs {
  rope_axes_desc_t rope;  // rotary_dim 0: nothing is rotated
  int32_t dtype;
  int32_t Hq, Hk, Hv;     // heads of q, k and v (Hv: append only)
  float sign;             // 1: forward, -1: gradient
  int64_t T;
  const void *q, *k, *v;
  void *q_out, *k_out;    // k_out: rotation only
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;  // elements
  const int32_t* positions;  // [num_axes, T]
  const float* inv_freq;
  // append: where new keys and values go
  void *k_cache, *v_cache;
  const int32_t *page_table, *seq_lens, *cu_new;
  int32_t B, table_width, page_shift;
  int64_t num_pages;
};
int launch_rope(const RopeArgs& a, void* stream);
int launch_append(const RopeArgs& a, void* stream);

struct PagedArgs {
  const void *q, *k_cache, *v_cache;
  void* out;
  float* lse;  // [Hq, T] or null
  const int32_t *page_table, *seq_lens, *cu_new;
  int64_t q_stride;  // elements
  int64_t num_pages;
  int32_t dtype, B, T, Hq, Hkv, D, group, table_width, page_shift;
  float scale;
};
int launch_paged_attn(const PagedArgs& a, void* stream);

}  // namespace pa

struct paged_attn_plan {
  paged_attn_desc_t desc;
  int32_t page_shift = 0;
  size_t ws_bytes = 0;
};
