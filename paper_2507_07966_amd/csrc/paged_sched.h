// How a call of paged_attn_forward is divided among its workgroups.  Lengths are known on the device only, so every workgroup works
// this out for itself from the lengths (and the host does the same for tests): plain integer arithmetic, no memory besides the
// two arrays.
//
// The work is a line.  A SEGMENT is a sequence with its new rows (and, with shared pages, one more for the shared
// keys, whose rows are those of all sequences); segments follow each other, in a segment the kv heads, in a head the blocks
// of `block_rows` stacked rows m = i * group + (h % group).  A block costs its keys plus START_KEYS for starting and
// ending it; the line is cut into equal shares, one a workgroup, and a block that a cut falls into becomes PIECES over
// disjoint ranges of its key tiles, whose partial results are merged.  Cutting by length on the device is what makes
// one launch fit all lengths: a call with one long sequence and many short ones keeps every compute unit busy to the end.
#pragma once

#include <cstdint>

#define PA_HD __host__ __device__ inline __attribute__((always_inline))

namespace pa {

struct PagedShape {
  int32_t B, T, Hkv, group;
  int32_t block_rows, tile_keys;
  int32_t block_tokens; // block_rows / group
  int32_t capacity;     // tokens that a row of the page table can name
  int32_t shared;       // leading keys of all sequences that form a segment of their own (whole pages); 0: none
  int32_t start_keys;   // cost of a block beside its keys
  int32_t min_share;    // keys: a smaller share is not worth a workgroup and a merge
  double inv_groups;    // 1 / workgroups
  float inv_group;      // 1 / group
  int32_t causal_cuts;  // cuts keep out of the tiles whose first key some row of the block does not see
};

struct Segment {
  int32_t token0, tokens;  // packed rows
  int32_t key0;            // first key
  int32_t blocks;          // of one kv head
  int64_t first_pos;       // position of the first token; shared keys: the last key's, every row sees all of them
  int32_t first_cost, more_cost;  // of block 0, and by how much each next one costs more
  int64_t cost;            // of one kv head
};

// x / group for 0 <= x < 2^20: half a step away from the next integer, fp32 rounding does not matter
PA_HD int32_t group_of(const PagedShape& s, int32_t x) { return (int32_t)(((float)x + 0.5f) * s.inv_group); }

// What a workgroup covers of a block: its key tiles [tile0, tile1).
struct Piece {
  int32_t block, tile0, tile1, key_end;
  bool whole;
};

PA_HD int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }
PA_HD int64_t blocks_cost(const Segment& g, int32_t n) {
  return (int64_t)n * g.first_cost + (g.more_cost ? g.more_cost * ((int64_t)n * (n - 1) / 2) : 0);
}
// a / b for a >= 0, b > 0 and a quotient below 2^31.  The compiler's 64-bit division is hundreds of instructions, which a workgroup runs
// (and fetches) once, before its first load: the quotient is guessed in fp64, off by at most one, and put right.
PA_HD int32_t div_small(int64_t a, int64_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
  const double d = (double)b;
  double r = __builtin_amdgcn_rcp(d);
  r = __builtin_fma(__builtin_fma(-d, r, 1.0), r, r);
  const int32_t q = (int32_t)((double)a * r);
  const int64_t rest = a - q * b;
  return rest < 0 ? q - 1 : rest >= b ? q + 1 : q;
#else
  return (int32_t)(a / b);
#endif
}

PA_HD Segment make_segment(const PagedShape& s, int64_t token0, int64_t tokens, int64_t first_pos, int64_t key0, int64_t keys,
                           int64_t more) {
  Segment g;
  g.token0 = (int32_t)token0;
  g.tokens = (int32_t)tokens;
  g.key0 = (int32_t)key0;
  g.blocks = (int32_t)((uint32_t)(tokens * s.group + s.block_rows - 1) / (uint32_t)s.block_rows);
  g.first_pos = first_pos;
  g.first_cost = (int32_t)(s.start_keys + keys);
  g.more_cost = (int32_t)more;
  g.cost = blocks_cost(g, g.blocks);
  return g;
}
// Sequence b's new rows and its own keys; cu0, cu1 = cu_new[b], cu_new[b + 1], len = seq_lens[b], whatever they hold.
PA_HD Segment own_segment(const PagedShape& s, int64_t cu0, int64_t cu1, int64_t len) {
  const int64_t lo = clamp64(cu0, 0, s.T), hi = clamp64(cu1, 0, s.T);
  const int64_t first = len - cu1 + lo;
  const int32_t per_block = s.block_tokens;
  const int64_t before = clamp64(first, 0, s.capacity) - s.shared;
  return make_segment(s, lo, hi > lo ? hi - lo : 0, first, s.shared, (before > 0 ? before : 0) + per_block, per_block);
}
PA_HD Segment shared_segment(const PagedShape& s, int64_t cu_end) {
  return make_segment(s, 0, s.shared > 0 ? clamp64(cu_end, 0, s.T) : 0, s.shared - 1, 0, s.shared, 0);
}

// What a call takes as shared: whole pages, within the table.
PA_HD int32_t whole_pages(const PagedShape& s, int32_t shared_len, int32_t page_shift) {
  return (int32_t)clamp64(shared_len, 0, s.capacity) & ~((1 << page_shift) - 1);
}

// Keys [key0, end) that the rows of a block see, one past the table included: it has no page and makes its rows NaN.
PA_HD int32_t block_key_end(const PagedShape& s, const Segment& g, bool shared, int32_t block) {
  if (shared) return s.shared;
  const int64_t rows = (int64_t)g.tokens * s.group, last = (int64_t)(block + 1) * s.block_rows;
  const int64_t i = (uint32_t)((last < rows ? last : rows) - 1) / (uint32_t)s.group;
  const int64_t end = clamp64(g.first_pos + i + 1, 0, (int64_t)s.capacity + 1);
  return (int32_t)(end > g.key0 ? end : g.key0);
}
// The tile at which a cut at cost x of a block that costs [c0, c1) falls.  Both sides of a cut compute it alike.
PA_HD int32_t cut_tile(const PagedShape& s, const Segment& g, bool shared, int32_t block, int64_t x, int64_t c0, int64_t c1, int32_t tiles) {
  if (x <= c0) return 0;
  if (x >= c1) return tiles;
  const int32_t t = div_small((x - c0) * tiles, c1 - c0);
  if (s.causal_cuts && !shared) {
    const int64_t first = g.first_pos + (uint32_t)(block * s.block_rows) / (uint32_t)s.group;  // position of the block's first row
    if (t > 0 && g.key0 + (int64_t)t * s.tile_keys > first) return tiles;
  }
  return t;
}
PA_HD Piece make_piece(const PagedShape& s, const Segment& g, bool shared, int32_t block, int64_t c0, int64_t c1, int64_t x0, int64_t x1) {
  Piece p;
  p.block = block;
  p.key_end = block_key_end(s, g, shared, block);
  const int32_t tiles = (p.key_end - g.key0 + s.tile_keys - 1) / s.tile_keys;
  p.tile0 = cut_tile(s, g, shared, block, x0, c0, c1, tiles);
  p.tile1 = cut_tile(s, g, shared, block, x1, c0, c1, tiles);
  p.whole = x0 <= c0 && x1 >= c1;
  return p;
}
// The block of a kv head in which cost `rem` of that head lies.
PA_HD int32_t block_at(const Segment& g, int64_t rem) {
  int32_t lo = 0, hi = g.blocks - 1;
  if (g.more_cost == 0) return div_small(rem, g.first_cost);
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) / 2;
    if (blocks_cost(g, mid) <= rem) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// Shares of the line: `share` of cost each, `active` of them; workgroup w of `groups` takes share number position(w), such that
// neighbouring shares, which read the same keys, run on one XCD (workgroup w is dispatched to XCD w % xcds).
PA_HD int64_t share_of(const PagedShape& s, int64_t total) {
  const int64_t even = (int64_t)((double)total * s.inv_groups) + 1 + (total >> 50);  // at least total / groups
  return even > s.min_share ? even : s.min_share;
}
PA_HD int32_t position_of(int32_t w, int32_t active, int32_t xcds) {
  const int32_t per = (active + xcds - 1) / xcds;
  const int32_t p = (w % xcds) * per + w / xcds;
  return w / xcds < per && p < active ? p : -1;
}

}  // namespace pa
