// How a call of paged_attn_forward is divided among its workgroups.  Lengths are known on the device only, so every workgroup works
// this out for itself from the lengths (and the host does the same for tests): plain integer arithmetic, no memory besides the
// two arrays.
//
// The work is a line.  A SEGMENT is a sequence with its new rows (and, with shared pages, one more for the shared
// keys, whose rows are those of all sequences); segments follow each other, in a segment the kv heads, in a head the blocks
// of `block_rows` stacked rows m = i * group + (h % group).  A block costs its keys (half of them where a sequence has so few rows that half
// of the workgroup idles) plus what starting and ending it costs; the line is cut into equal shares, one a workgroup, and a block that a
// cut falls into becomes PIECES over disjoint ranges of its key tiles, whose partial results are merged.  Cutting by length on the device
// is what makes one launch fit all lengths: a call with one long sequence and many short ones keeps every compute unit busy to the end.
//
// Before its first load a workgroup can do nothing else than this, so it is kept short: cost is counted in units of
// 2^unit_shift keys, which the host chooses such that no call of its sizes exceeds 2^30 units (16 keys, but for calls beyond any real
// one), so that everything but the lengths themselves fits 32 bits, and a cut finds its tile without a division.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define PA_HD __host__ __device__ inline __attribute__((always_inline))
#else
#define PA_HD inline
#endif

namespace pa {

struct PagedShape {
  int32_t B, T, Hkv, group;
  int32_t block_rows, tile_shift;  // rows of a block, log2 of the keys of a tile
  int32_t capacity;     // tokens that a row of the page table can name
  int32_t shared;       // leading keys of all sequences that form a segment of their own (whole pages); 0: none
  int32_t unit_shift;
  int32_t start_cost;   // of a block beside its keys, in units
  int32_t growth;       // by how many keys a block of new tokens sees more than the one before it (a block's tokens), times 2^GROWTH_SHIFT
  int32_t min_share;    // units: a smaller share is not worth a workgroup and a merge
  int32_t half_rows;    // a sequence of at most so many rows has a block of half the cost a key
  int32_t causal_cuts;  // cuts keep out of the tiles whose first key some row of the block does not see
  float per_group;      // a little more than 1 / workgroups
  float inv_group;      // 1 / group
};

// A block's tokens, block_rows / group, are no whole number, and in a prefill from nothing the new tokens are most of the keys, so the growth
// is not rounded before it is summed: in units of 16 keys it was 32 for 36.6 tokens and 0 for 12.8, and the fullest share of 4,096 tokens from
// nothing had 2.95 (32 + 1 heads, bf16) and 2.38 (8 + 2, fp32) times the mean of the tiles; now 1.11 and 1.05 (355 -> 185 us; 2,048
// tokens of 8 + 2 heads in fp32: 244 -> 123).
constexpr int GROWTH_SHIFT = 12;

struct Segment {
  int32_t token0, tokens;  // packed rows
  int32_t key0;            // first key
  int32_t blocks;          // of one kv head
  int32_t first_pos;       // position of the first token
  int32_t first_cost, growth;  // cost of block 0; as in PagedShape, 0 for the shared keys
  int32_t cost;            // of one kv head; -1: cu_new falls here, and the call does nothing
};

// What a workgroup covers of a block: its key tiles [tile0, tile1).
struct Piece {
  int32_t tile0, tile1, key_end;
  bool whole;
};

PA_HD int64_t clamp64(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }
// Of a head's first n blocks.  (n * growth is below 2^37, as a sequence has at most 2^24 tokens, and n below 2^27: 2^63 is not reached.)
PA_HD int32_t blocks_cost(const PagedShape& s, const Segment& g, int32_t n) {
  return n * g.first_cost + (n > 1 ? (int32_t)((int64_t)n * (n - 1) / 2 * g.growth >> (GROWTH_SHIFT + s.unit_shift)) : 0);
}
// a / b for 0 <= a < 2^31, b > 0 and a quotient below 2^20: guessed in fp32, off by at most one, and put right
PA_HD int32_t div_small(int32_t a, int32_t b) {
#if defined(__HIP_DEVICE_COMPILE__)
  const int32_t q = (int32_t)((float)a * __builtin_amdgcn_rcpf((float)b));
  const int32_t rest = a - q * b;
  return rest < 0 ? q - 1 : rest >= b ? q + 1 : q;
#else
  return a / b;
#endif
}
// x / group for 0 <= x < 2^20: half a step away from the next integer, fp32 rounding does not matter
PA_HD int32_t group_of(const PagedShape& s, int32_t x) { return (int32_t)(((float)x + 0.5f) * s.inv_group); }

// log2 of the keys that cost a unit in this segment
PA_HD int32_t key_shift_of(const PagedShape& s, const Segment& g) {
  return s.unit_shift + ((uint32_t)g.tokens * (uint32_t)s.group <= (uint32_t)s.half_rows);
}
PA_HD Segment make_segment(const PagedShape& s, int32_t token0, int32_t tokens, int32_t first_pos, int32_t key0, int32_t keys, int32_t growth) {
  Segment g;
  g.token0 = token0;
  g.tokens = tokens;
  g.key0 = key0;
  const uint32_t rows = (uint32_t)tokens * (uint32_t)s.group;
  g.blocks = rows <= (uint32_t)s.block_rows ? (rows > 0) : (int32_t)((rows + s.block_rows - 1) / (uint32_t)s.block_rows);
  g.first_pos = first_pos;
  g.first_cost = s.start_cost + (keys >> key_shift_of(s, g));
  g.growth = growth;
  g.cost = blocks_cost(s, g, g.blocks);
  return g;
}
// Sequence b's new rows and its own keys; cu0, cu1 = cu_new[b], cu_new[b + 1], len = seq_lens[b], whatever they hold.  (A first position
// behind the table stays behind it, one so far below 0 that no row reaches 0 stays there.)
PA_HD Segment own_segment(const PagedShape& s, int32_t cu0, int32_t cu1, int32_t len) {
  const int32_t lo = (int32_t)clamp64(cu0, 0, s.T), hi = (int32_t)clamp64(cu1, 0, s.T);
  const int32_t first = (int32_t)clamp64((int64_t)len - cu1 + lo, -(1 << 30), s.capacity);
  const int32_t tokens = hi > lo ? hi - lo : 0, of_block = (s.growth + (1 << GROWTH_SHIFT) - 1) >> GROWTH_SHIFT;
  const int32_t keys = first + (tokens < of_block ? tokens : of_block) - s.shared;  // that block 0 sees
  Segment g = make_segment(s, lo, tokens, first, s.shared, keys > 0 ? keys : 0, s.growth);
  if (cu1 < cu0) g.cost = -1;  // sequences might overlap, and the line be longer than the unit allows for
  return g;
}
PA_HD Segment shared_segment(const PagedShape& s, int32_t cu_end) {
  return make_segment(s, 0, s.shared > 0 ? (int32_t)clamp64(cu_end, 0, s.T) : 0, 0, 0, s.shared, 0);
}
// What a call takes as shared: whole pages, within the table.
PA_HD int32_t whole_pages(const PagedShape& s, int32_t shared_len, int32_t page_shift) {
  return (int32_t)clamp64(shared_len, 0, s.capacity) & ~((1 << page_shift) - 1);
}

// A block's place on the line: costs [c0, c1), counted like x in the caller's way.
// `token`: of its first row, counted from the segment's first token; `row`: that row among its token's rows.
struct Block {
  int32_t c0, c1, rows, token, row;
};
PA_HD Block make_block(const PagedShape& s, const Segment& g, int32_t head_start, int32_t block) {
  Block b;
  b.c0 = head_start + blocks_cost(s, g, block);
  b.c1 = head_start + blocks_cost(s, g, block + 1);
  const uint32_t row0 = (uint32_t)block * (uint32_t)s.block_rows, left = (uint32_t)g.tokens * (uint32_t)s.group - row0;
  b.rows = left < (uint32_t)s.block_rows ? (int32_t)left : s.block_rows;
  b.token = block ? (int32_t)(row0 / (uint32_t)s.group) : 0;
  b.row = (int32_t)(row0 - (uint32_t)b.token * (uint32_t)s.group);
  return b;
}
// The piece of a block between x0 and x1.  The rows of a block see the keys [key0, key_end), one past the table included: it has no page and
// makes them NaN.  A cut at cost x falls on the tile that x - c0 - start_cost units lead to; both sides of a cut compute it alike.
PA_HD Piece make_piece(const PagedShape& s, const Segment& g, bool shared, const Block& b, int32_t x0, int32_t x1) {
  Piece p;
  p.key_end = s.shared;
  int32_t first_cut = 0x7fffffff;  // tiles from this one on are not cut apart
  if (!shared) {
    const int32_t last = g.first_pos + b.token + group_of(s, b.row + b.rows - 1);
    const int32_t end = last >= s.capacity ? s.capacity + 1 : last + 1;
    p.key_end = end > g.key0 ? end : g.key0;
    if (s.causal_cuts) {
      const int32_t seen = g.first_pos + b.token - g.key0;  // of the block's first row, beyond key0
      first_cut = seen < 0 ? 0 : seen >> s.tile_shift;
    }
  }
  const int32_t tiles = (p.key_end - g.key0 + (1 << s.tile_shift) - 1) >> s.tile_shift;
  p.whole = x0 <= b.c0 && x1 >= b.c1;
  p.tile0 = 0;
  p.tile1 = tiles;
  if (!p.whole) {
    const int32_t shift = key_shift_of(s, g) - s.tile_shift;
    auto tile = [&](int32_t x) {
      const int64_t u = x - b.c0 - s.start_cost;
      const int64_t t = u <= 0 ? 0 : shift >= 0 ? u << shift : u >> -shift;
      return (int32_t)(t > tiles || (t > first_cut && t > 0) ? tiles : t);
    };
    if (x0 > b.c0) p.tile0 = tile(x0);
    if (x1 < b.c1) p.tile1 = tile(x1);
  }
  return p;
}
// The block of a kv head in which cost `rem` of that head lies.
PA_HD int32_t block_at(const PagedShape& s, const Segment& g, int32_t rem) {
  if (g.blocks <= 1) return 0;
  if (g.growth == 0) return (int32_t)((uint32_t)rem / (uint32_t)g.first_cost);
  int32_t lo = 0, hi = g.blocks - 1;
  while (lo < hi) {
    const int32_t mid = (lo + hi + 1) >> 1;
    if (blocks_cost(s, g, mid) <= rem) lo = mid; else hi = mid - 1;
  }
  return lo;
}
// Shares of the line: `share` units of cost each, `active` of them; workgroup w takes share number position_of(w), such that
// neighbouring shares, which read the same keys, run on one XCD (workgroup w is dispatched to XCD w % 2^xcd_shift).
PA_HD int32_t share_of(const PagedShape& s, int32_t total) {
  const int32_t even = (int32_t)((float)total * s.per_group) + 1;  // at least total / workgroups
  return even > s.min_share ? even : s.min_share;
}
PA_HD int32_t active_of(int32_t total, int32_t share) { return div_small(total + share - 1, share); }
PA_HD int32_t position_of(int32_t w, int32_t active, int32_t xcd_shift) {
  const int32_t per = (active + (1 << xcd_shift) - 1) >> xcd_shift, in = w >> xcd_shift;
  const int32_t p = (w & ((1 << xcd_shift) - 1)) * per + in;
  return in < per && p < active ? p : -1;
}

}  // namespace pa
