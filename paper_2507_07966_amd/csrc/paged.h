// Internal declarations of the sampling phase: rotary positions, paged cache and attention over pages.
#pragma once

#include <cstddef>
#include <cstdint>

#include "paged_attn.h"
#include "paged_sched.h"

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

// A block whose keys were cut into pieces: pieces first .. last (numbers of shares) cover it.
struct PagedCut {
  int32_t token0, tokens, head, block;  // as in Segment and Piece; tokens 0: the share begins no block that it does not end
  int32_t first, last;
};
// What workgroup 0 tells the merge about the line.
struct PagedLine {
  int32_t share, active, shared;
};

struct PagedArgs {
  const void *q, *k_cache, *v_cache;
  void* out;
  float* lse;  // [Hq, T] or null
  const int32_t *page_table, *seq_lens, *cu_new, *shared_len;
  int64_t q_stride;  // elements
  int64_t num_pages;
  int32_t dtype, D, Hq, table_width, page_shift;
  float scale;
  PagedShape shape;        // `shared` is read on the device
  int32_t groups, xcd_shift;  // workgroups, and log2 of the XCDs that they are laid out over
  int32_t blocks16;        // few rows: 16-row blocks of a block
  // workspace
  PagedLine* line;
  int32_t* seg_start;      // [B + 2] cost at which segment i begins (with shared keys only: segment 0 is theirs)
  PagedCut* cuts;          // [groups]
  float* slots;            // [2 * groups][block_rows][D] fp32 partial outputs: of the block that share i continues (2 i) and
  float* slot_lse;         //   of the one that it begins and does not end (2 i + 1); [2 * groups][block_rows]
  float* rows;             // with shared keys, [2][T * Hq][D]: partials of whole blocks, own keys and shared ones
  float* rows_lse;         // [2][T * Hq]
};
int launch_paged_rows(const PagedArgs& a, void* stream);   // calls of few rows a sequence, and fp32
// Its wavefronts, and the bytes of keys (and of values) that one of them has in a step: together the keys of a tile
constexpr int PAGED_ROWS_WAVES = 4, PAGED_ROWS_HALF_STAGE = 8192;
inline int paged_rows_tile_shift(int32_t dtype, int32_t D) {
  int shift = 0;
  while ((D * (dtype == PA_BF16 ? 2 : 4)) << shift < PAGED_ROWS_WAVES * PAGED_ROWS_HALF_STAGE) ++shift;
  return shift;
}
constexpr int PAGED_CHUNK_ROWS = 256, PAGED_CHUNK_TILE_SHIFT = 6;
int launch_paged_chunk(const PagedArgs& a, void* stream);  // bf16 calls of many rows a sequence
int launch_paged_merge(const PagedArgs& a, void* stream);

}  // namespace pa

struct paged_attn_plan {
  paged_attn_desc_t desc;
  int32_t page_shift = 0;
  int32_t num_cu = 256, xcd_shift = 3;
  int32_t group = 1;
  // workspace: byte offsets
  size_t off_seg_start = 0, off_cuts = 0, off_slot_lse = 0, off_slots = 0, off_rows_lse = 0, off_rows = 0, ws_bytes = 0;
};
