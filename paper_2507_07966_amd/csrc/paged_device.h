// Device side of the schedule of paged_sched.h, and small helpers of the kernels that attend over pages.
#pragma once

#include <hip/hip_runtime.h>

#include "mfma_tiles.h"
#include "paged.h"

namespace pa {

// Exchange between lane l and lane l^32 (v_permlane32_swap; the results are read through named temporaries, as in the
// prefill kernels), and reductions over the four lanes l, l^16, l^32, l^48 that hold one query column.
__device__ inline void pair_exchange(float x, float& lo, float& hi) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const unsigned r0 = r[0], r1 = r[1];
  lo = __uint_as_float(r0);
  hi = __uint_as_float(r1);
}
__device__ inline float quad_max(float x) {
  float a, b;
  pair_exchange(fmaxf(x, __shfl_xor(x, 16)), a, b);
  return fmaxf(a, b);
}
__device__ inline float quad_sum(float x) {
  float a, b;
  pair_exchange(x + __shfl_xor(x, 16), a, b);
  return a + b;
}

// Swizzle of row-major tiles that are read both as 16-byte operands (16 consecutive rows at one 16-byte chunk) and transposed in 16 x 16
// blocks (ds_read_b64_tr_b16: lane l of a group of 16 reads 8 bytes of row 4 g + l / 4, so half a wavefront reads 32 bytes of 8
// consecutive rows): chunk c of row r is stored at c ^ swizzle16(r), which puts the pieces of either access on different banks.
__device__ inline int swizzle16(int row, int row_bytes) {
  const int low = ((row >> 1) & 2) | ((row >> 3) & 1);
  return row_bytes == 256 ? ((row & 3) << 2) | low : ((row & 2) << 1) | low;
}

// Wait until at most N of this wavefront's vector memory operations are under way (loads to LDS complete in order), or until its
// reads of LDS have returned.  The compiler keeps memory accesses on their side of it.
template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// A barrier that does not wait for loads to LDS, as __syncthreads() does: the caller has waited for those that the workgroup is to see.
__device__ inline void barrier_with_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ inline void wait_lds_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Lengths, tables and the like: nothing writes them while a kernel runs, which the address space says, so that uniform reads are scalar.
__device__ inline int32_t read_const(const int32_t* p, int64_t i) {
  typedef const __attribute__((address_space(4))) int32_t* Const;
  return ((Const)p)[i];
}

// Where a row of a block's result goes: the call's output, or an fp32 partial.
struct Place {
  void* row;
  float* lse;
  bool partial;
};
template <typename T>
__device__ inline void write_row(const Place& p, int ch, mt::f32x4 v) {
  if (p.partial) {
    *reinterpret_cast<mt::f32x4*>(static_cast<float*>(p.row) + ch) = v;
  } else {
    typedef T T4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T4*>(static_cast<T*>(p.row) + ch) = __builtin_convertvector(v, T4);
  }
}

__device__ inline int32_t shared_keys(const PagedArgs& a) {
  if (!a.shared_len) return 0;
  return whole_pages(a.shape, read_const(a.shared_len, 0), a.page_shift);
}
// What segment i is made from: read before `shared` is known, so that the reads do not wait for each other.
struct Lengths {
  int32_t cu0, cu1, len;
};
__device__ inline Lengths read_lengths(const PagedArgs& a, int i) {
  const int with = a.shared_len ? 1 : 0;
  if (i < with) return Lengths{0, read_const(a.cu_new, a.shape.B), 0};
  return Lengths{read_const(a.cu_new, i - with), read_const(a.cu_new, i - with + 1), read_const(a.seq_lens, i - with)};
}
__device__ inline Segment segment_of(const PagedArgs& a, const PagedShape& s, int i, const Lengths& l) {
  return a.shared_len && i == 0 ? shared_segment(s, l.cu1) : own_segment(s, l.cu0, l.cu1, l.len);
}
__device__ inline Segment load_segment(const PagedArgs& a, const PagedShape& s, int i) { return segment_of(a, s, i, read_lengths(a, i)); }

// The last key that a new token sees, at most the one behind the table; -1: none.
__device__ inline int32_t row_limit(const PagedShape& s, const Segment& g, int32_t token) {
  const int32_t pos = g.first_pos + token;
  return pos < 0 ? -1 : pos < s.capacity ? pos : s.capacity;
}

// Where some consecutive rows of a head are in the cache.  They lie in one page; the buffer descriptor's range ends with the last row that
// exists, or is empty, and LDS receives zeros behind it.
struct Rows {
  int64_t off;  // bytes from the cache's begin
  int32_t bytes;
};
// `key`: the first of `count` rows of `row_bytes`; keys from `end` on do not exist.  `first_lost` becomes the smallest key without a page.
__device__ inline Rows find_rows(const PagedArgs& a, int32_t page, uint32_t page_bytes, int64_t head_bytes, int32_t key, int32_t end,
                                 int32_t count, int32_t row_bytes, int32_t& first_lost) {
  const int32_t left = end - key < count ? end - key : count;
  const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
  if (!ok && left > 0) first_lost = key < first_lost ? key : first_lost;
  return Rows{(int64_t)((uint64_t)(uint32_t)page * page_bytes) + head_bytes + (key & ((1 << a.page_shift) - 1)) * row_bytes,
              ok && left > 0 ? left * row_bytes : 0};
}
// 16 bytes a lane straight to LDS (lane l's land at dst + 16 l) that the compiler does not know of.  It waits for every load to LDS that it
// knows of before the next read of LDS that may overlap it, and it cannot tell the buffers of a ring apart: a kernel that has later tiles
// under way while it reads an earlier one counts its loads itself (wait_loads).  s_nop 4: a descriptor that a vector instruction
// has just written to scalar registers may be read by a buffer instruction five states later, m0 one.
__device__ inline void load_chunk_to_lds_uncounted(const void* cache, const Rows& r, unsigned char* dst, unsigned lane_byte_offset) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint64_t base = (uint64_t)(uintptr_t)cache + (uint64_t)r.off;
  const mt::i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)base), __builtin_amdgcn_readfirstlane((int)(base >> 32) & 0xffff),
                          __builtin_amdgcn_readfirstlane(r.bytes), 0x00020000};
  const unsigned lds = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(PA_LDS_PTR(unsigned char))dst);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(lane_byte_offset), "s"(rsrc) : "memory", "m0");
#endif
}
#if defined(__HIP_DEVICE_COMPILE__)
__device__ inline mt::rsrc_t rows_rsrc(const void* cache, const Rows& r) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(cache) + r.off), 0, r.bytes, 0x00020000);
}
#else
__device__ inline mt::rsrc_t rows_rsrc(const void*, const Rows&) { return {}; }
#endif
// The page of `key` in a row of the page table (keys behind the table: of its last column, they do not exist)
__device__ inline int32_t page_of(const PagedArgs& a, const int32_t* table, int32_t key) {
  const int32_t idx = key >> a.page_shift;
  return read_const(table, idx < a.table_width ? idx : a.table_width - 1);
}

// A workgroup's way along its share: one piece of a block at a time.  All members are uniform.
struct Walk {
  PagedShape shape;
  Segment seg;
  Block block;
  int32_t seg_index, segments, head, block_index;
  int32_t head_start;  // where the kv head's blocks begin on the line
  int32_t x, x_end;    // what is left of the share
  int32_t share, position;
  int32_t table_row;   // of the page table
  int32_t first_seq;   // the first sequence with new tokens: shared keys are read through its row
  bool shared;         // the segment is that of the shared keys

  __device__ bool more() const { return x < x_end; }
  __device__ void enter(const PagedArgs& a) {
    shared = a.shared_len && seg_index == 0;
    table_row = shared ? first_seq : seg_index - (a.shared_len ? 1 : 0);
  }
  __device__ Piece piece() {
    block = make_block(shape, seg, head_start, block_index);
    return make_piece(shape, seg, shared, block, x, x_end);
  }
  __device__ void next(const PagedArgs& a) {
    x = x_end < block.c1 ? x_end : block.c1;
    if (x >= x_end) return;
    if (++block_index < seg.blocks) return;
    block_index = 0;
    head_start += seg.cost;
    if (++head < shape.Hkv) return;
    head = 0;
    do {
      seg = load_segment(a, shape, ++seg_index);  // there is one more with work: x < x_end
    } while (seg.cost == 0 && seg_index + 1 < segments);
    enter(a);
  }
  // The token (counted from the segment's first) and the query head of the block's row r.
  __device__ int32_t row_token(int32_t r) const { return block.token + group_of(shape, block.row + r); }
  __device__ int32_t row_head(int32_t r, int32_t tok) const { return head * shape.group + block.row + r - (tok - block.token) * shape.group; }
  __device__ Place place(const PagedArgs& a, const Piece& p, int r) const {
    if (!p.whole) {
      const int64_t row = (2 * position + (x == block.c0 ? 1 : 0)) * shape.block_rows + r;
      return Place{a.slots + row * a.D, a.slot_lse + row, true};
    }
    const int32_t tok = row_token(r);
    const int64_t t = seg.token0 + tok, h = row_head(r, tok);
    if (!a.shared_len)
      return Place{static_cast<char*>(a.out) + (t * a.Hq + h) * a.D * (a.dtype == PA_BF16 ? 2 : 4), a.lse ? a.lse + h * shape.T + t : nullptr, false};
    const int64_t row = ((shared ? (int64_t)shape.T : 0) + t) * a.Hq + h;
    return Place{a.rows + row * a.D, a.rows_lse + row, true};
  }
  // Thread 0 notes for the merge a block that this share begins and does not end.
  __device__ void note_cut(const PagedArgs& a) const {
    if (threadIdx.x == 0 && x == block.c0 && x_end < block.c1)
      a.cuts[position] = PagedCut{seg.token0, seg.tokens, head, block_index, position, div_small(block.c1 - 1, share)};
  }
};

// Finds the workgroup's share; false: it has none.  Every thread of the workgroup calls it.
template <int THREADS>
__device__ inline bool begin_walk(const PagedArgs& a, Walk& w) {
  constexpr int WAVES = THREADS / 64;
  __shared__ uint32_t wave_cost[WAVES], found_start;  // (unsigned: where cu_new falls the sums mean nothing)
  __shared__ Segment found;
  __shared__ int32_t found_segment, first_seq, falls;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Lengths mine{0, 0, 0};
  if (tid < a.shape.B + (a.shared_len ? 1 : 0)) mine = read_lengths(a, tid);
  w.shape = a.shape;
  w.shape.shared = shared_keys(a);
  const int with = a.shared_len ? 1 : 0;
  w.segments = a.shape.B + with;
  if (tid == 0) {
    first_seq = 0x7fffffff;
    falls = 0;
  }
  __syncthreads();
  // Two rounds over the segments where they are more than the threads: the sum of all costs, then the share's segment.
  uint32_t total = 0, start = 0, cost = 0;
  Segment g;
  const int lanes = w.segments < 64 ? w.segments : 64;
  auto round = [&](int base) {  // start and cost of segment base + tid; total: those before base, and then with this round's
    const int i = base + tid;
    cost = 0;
    if (i < w.segments) {
      g = segment_of(a, w.shape, i, base == 0 ? mine : read_lengths(a, i));
      if (g.cost < 0) falls = 1;
      cost = g.cost < 0 ? 0u : (uint32_t)(w.shape.Hkv * g.cost);
      if (i >= with && cost > 0) atomicMin(&first_seq, i - with);
    }
    uint32_t sum = cost;
    for (int d = 1; d < lanes; d *= 2) {
      const uint32_t up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    if (lane == lanes - 1) wave_cost[wave] = sum;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int v = 0; v < WAVES; ++v) {
      before += v < wave ? wave_cost[v] : 0;
      all += wave_cost[v];
    }
    start = total + before + sum - cost;
    total += all;
    __syncthreads();
  };
  for (int base = 0; base < w.segments; base += THREADS) {
    round(base);
    if (blockIdx.x == 0 && with && base + tid < w.segments) a.seg_start[base + tid] = (int32_t)start;
  }
  const int32_t length = __builtin_amdgcn_readfirstlane(falls ? 0 : (int32_t)total);
  w.share = share_of(w.shape, length);
  const int32_t active = active_of(length, w.share);
  if (blockIdx.x == 0 && tid == 0) *a.line = PagedLine{w.share, active, w.shape.shared};
  w.position = position_of(blockIdx.x, active, a.xcd_shift);
  if (w.position < 0) return false;
  w.x = w.position * w.share;
  w.x_end = w.x + w.share < length ? w.x + w.share : length;
  if (w.segments > THREADS) total = 0;
  for (int base = 0; base < w.segments; base += THREADS) {
    if (w.segments > THREADS) round(base);
    if (start <= (uint32_t)w.x && (uint32_t)w.x < start + cost) {
      found_segment = base + tid;
      found_start = start;
      found = g;
    }
  }
  __syncthreads();
  w.seg_index = __builtin_amdgcn_readfirstlane(found_segment);
  w.first_seq = __builtin_amdgcn_readfirstlane(first_seq < a.shape.B ? first_seq : a.shape.B - 1);
  w.seg.token0 = __builtin_amdgcn_readfirstlane(found.token0);
  w.seg.tokens = __builtin_amdgcn_readfirstlane(found.tokens);
  w.seg.key0 = __builtin_amdgcn_readfirstlane(found.key0);
  w.seg.blocks = __builtin_amdgcn_readfirstlane(found.blocks);
  w.seg.first_pos = __builtin_amdgcn_readfirstlane(found.first_pos);
  w.seg.first_cost = __builtin_amdgcn_readfirstlane(found.first_cost);
  w.seg.growth = __builtin_amdgcn_readfirstlane(found.growth);
  w.seg.cost = __builtin_amdgcn_readfirstlane(found.cost);
  const int32_t seg_start = __builtin_amdgcn_readfirstlane((int32_t)found_start);
  w.head = __builtin_amdgcn_readfirstlane(div_small(w.x - seg_start, w.seg.cost));
  w.head_start = seg_start + w.head * w.seg.cost;
  w.block_index = __builtin_amdgcn_readfirstlane(block_at(w.shape, w.seg, w.x - w.head_start));
  w.enter(a);
  if (tid == 0) a.cuts[w.position] = PagedCut{0, 0, 0, 0, 0, 0};
  return true;
}

}  // namespace pa
