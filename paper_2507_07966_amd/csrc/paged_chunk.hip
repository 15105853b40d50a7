// Attention of new tokens over their pages for chunks (bf16): blocks of 256 stacked rows.
//
// Bound: bf16 MFMA.  A block is 256 rows m = i * group + (h % group) of one kv head and sequence, 32 a wavefront, two wavefronts a SIMD;
// tiles of 64 keys go to LDS once for all of them, room for four of K and of V (one that is read, three under way), one barrier a tile.  Products, operand order and the
// interleave of one tile's softmax with the product before are those of the prefill kernels (v_mfma_f32_16x16x32_bf16 on transposed
// scores); what differs:
//   - Keys come from pages.  A wavefront loads 8 rows of a tile; they lie in one page (page sizes are multiples of 16), whose
//     number is read into scalar registers one tile ahead, and the buffer descriptor is made for them: 64-bit address, range up to the
//     last key, so that nothing past it is read and LDS holds zeros there.  A row of the block that sees a key without a page, which is one
//     whose limit is not below the smallest such key, becomes NaN at the end.
//   - V is read transposed from row-major tiles (ds_read_b64_tr_b16): a paged cache has no images of its values.
//   - The reference of the softmax is the maximum of a row's first tile, with no search afterwards; a tile's sum tells when some
//     probability left the safe range.  Then the block is done again with its true maxima, which a pass over the
//     scores alone finds first: one loop serves both, and no code that rescales accumulators takes registers from it.  That pass has one
//     tile under way at a time.  Where every block is done again (scores that grow by more than 11 along a sequence, or one key far above
//     the others in its middle) a call takes 2.3 ... 2.4 times as long: 881 -> 2,140 us for the first call below, 139 -> 318 for the second.
//   - A workgroup takes a share of the line of paged_sched.h: whole blocks, and parts of the two that its ends cut.
//
// Measured: the last 2,048 tokens of a sequence of 34,816 (28 + 4 heads of 128): 0.87 ... 0.92 ms, 1.1 PFLOP/s, the matrix pipe busy 54 %
// of the cycles (the prefill kernels, whose values are stored as images, take 0.82).  24 chunks of 19 ... 294 tokens, 14 + 2 heads
// of 64: 134 us, 0.65 PFLOP/s: 4.6 other vector instructions to an MFMA that is half as long, matrix pipe busy 30 %, wavefronts waiting
// 32 %: 511 pieces, each of which begins with nothing under way.  No LDS
// bank conflicts.  Loads issued between the MFMAs instead of at a tile's end: 905 ... 917 us (897); half of the wavefronts half a tile behind
// the others, with a buffer more: 902 (874) and 147 (132); wave priorities make no difference.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "common.h"
#include "mfma_tiles.h"
#include "paged.h"
#include "paged_device.h"

namespace pa {
namespace {

using namespace mt;

constexpr int NQ = 2, WAVES = 8, THREADS = WAVES * 64, ROWS_PER_WAVE = 16 * NQ, ROWS = WAVES * ROWS_PER_WAVE;
static_assert(ROWS == PAGED_CHUNK_ROWS && TILE == 1 << PAGED_CHUNK_TILE_SHIFT, "the schedule's blocks and tiles");
constexpr float SAFE_SUM = 65536.0f;  // a lane's sum of a tile's probabilities below this keeps fp32 and bf16 far from overflow
constexpr int RING = 4;               // LDS operand reads ahead of the MFMAs that use them

template <int D>
__global__ __launch_bounds__(THREADS, 1) void paged_chunk_kernel(const PagedArgs a) {
  constexpr int ROWB = 2 * D, TILE_BYTES = TILE * ROWB, KS = D / 32, CB = D / 16;
  constexpr int LOADS = TILE_BYTES / 1024 / WAVES;  // 1 KiB loads of a wavefront, of K and of V
  constexpr int LANES_PER_ROW = ROWB / 16, ROWS_PER_LOAD = 1024 / ROWB;
  constexpr int WAVE_KEYS = TILE / WAVES;           // rows of a tile that a wavefront loads
  constexpr int AHEAD = 3, BUFS = AHEAD + 1;  // tiles under way beside the one that is read
  constexpr int VBUF = BUFS * TILE_BYTES;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * BUFS * TILE_BYTES];
  __shared__ int32_t gave_up[WAVES], wave_lost[WAVES];

  Walk walk;
  if (!begin_walk<THREADS>(a, walk)) return;
  const PagedShape& shape = walk.shape;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float c_log2 = a.scale * 1.4426950408889634f;

  int koff[KS], vtr[CB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) koff[ks] = l16 * ROWB + (((4 * ks + g4) ^ swizzle_term(l16, ROWB)) << 4);
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int r = 4 * g4 + (l16 >> 2);
    vtr[cb] = r * ROWB + (((2 * cb + ((l16 & 3) >> 1)) ^ swizzle16(r, ROWB)) << 4) + (l16 & 1) * 8;
  }
  unsigned kload[LOADS], vload[LOADS];  // byte offset of this lane's 16 bytes in the wavefront's rows of the cache
#pragma unroll
  for (int n = 0; n < LOADS; ++n) {
    const int in = n * ROWS_PER_LOAD + lane / LANES_PER_ROW, row = wave * WAVE_KEYS + in;
    kload[n] = (unsigned)(in * ROWB + (((lane % LANES_PER_ROW) ^ swizzle_term(row, ROWB)) << 4));
    vload[n] = (unsigned)(in * ROWB + (((lane % LANES_PER_ROW) ^ swizzle16(row, ROWB)) << 4));
  }

  for (; walk.more(); walk.next(a)) {
    const Piece p = walk.piece();
    const Segment& seg = walk.seg;
    const int block_rows = walk.block.rows;
    const int32_t* const table = a.page_table + (int64_t)walk.table_row * a.table_width;
    const int first_key = seg.key0 + p.tile0 * TILE, tiles = p.tile1 - p.tile0;

    // ---- this lane's two query columns
    // A wavefront without rows only loads: with at most half of a block's rows every SIMD has one wavefront left that computes, and a tile takes
    // about half the time (a token a sequence in such blocks: 271 -> 203 us, the rate of memory), which the schedule counts on.
    const bool idle = wave * ROWS_PER_WAVE >= block_rows;
    bf16x8 Q[NQ][KS];
    int limit[NQ];  // last key that column nq sees
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = wave * ROWS_PER_WAVE + nq * 16 + l16;
      const __bf16* row = nullptr;
      limit[nq] = 0x7fffffff;
      if (r < block_rows) {
        const int tok = walk.row_token(r);
        row = static_cast<const __bf16*>(a.q) + (int64_t)(seg.token0 + tok) * a.q_stride + walk.row_head(r, tok) * D + 8 * g4;
        limit[nq] = row_limit(shape, seg, tok);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) Q[nq][ks] = row ? *reinterpret_cast<const bf16x8*>(row + 32 * ks) : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
    // keys up to this one are seen by every row of the wavefront (positions do not fall from row to row)
    const int first_limit = __builtin_amdgcn_readfirstlane(limit[0]);

    // Where a wavefront's rows of tile t are: found for K, and used for V one step later.  The page number is read two steps before.
    const uint32_t page_bytes = ((uint32_t)shape.Hkv << a.page_shift) * (uint32_t)ROWB;
    const int64_t head_bytes = ((int64_t)walk.head << a.page_shift) * ROWB;
    const int wave_key = first_key + wave * WAVE_KEYS;
    int last_key = first_key + tiles * TILE < p.key_end ? first_key + tiles * TILE : p.key_end;
    int first_lost = last_key > shape.capacity ? shape.capacity : 0x7fffffff;  // smallest key without a page: rows that see it become NaN
    last_key = last_key < shape.capacity ? last_key : shape.capacity;
    auto look_up = [&](int t) { return page_of(a, table, wave_key + t * TILE); };
    auto source = [&](int t, int page) {
      return find_rows(a, page, page_bytes, head_bytes, wave_key + t * TILE, last_key, WAVE_KEYS, ROWB, first_lost);
    };
    // Every step issues as many loads as every other (empty ones behind the last tile), so that a wait can count them.
    auto issue_k = [&](const Rows& from, int buf) {  // buf: byte offset of the buffer, K's and V's alike
      unsigned char* const dst = smem + buf + wave * LOADS * 1024;
#pragma unroll
      for (int n = 0; n < LOADS; ++n) load_chunk_to_lds_uncounted(a.k_cache, from, dst + n * 1024, kload[n]);
    };
    auto issue_v = [&](const Rows& from, int buf) {
      unsigned char* const dst = smem + VBUF + buf + wave * LOADS * 1024;
#pragma unroll
      for (int n = 0; n < LOADS; ++n) load_chunk_to_lds_uncounted(a.v_cache, from, dst + n * 1024, vload[n]);
    };

    f32x4 O[CB][NQ];    // O^T: register i of block cb is channel 16 cb + 4 g4 + i of column nq
    f32x4 S[4][NQ];     // scores of the tile being soft-maxed: register i of block kb is key 16 kb + 4 g4 + i
    bf16x8 Pb[2][NQ];   // probabilities of the tile before, as the operand of its product with V
    float mref[NQ], lsum[NQ];
    bool bad = false;

    auto scores = [&](const unsigned char* kbuf) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) S[kb][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
      auto operand = [&](int t) { return lds_operand(kbuf + (t % 4) * 16 * ROWB + koff[t / 4]); };
      constexpr int OPS = 4 * KS;
      bf16x8 ka[RING];
#pragma unroll
      for (int t = 0; t < RING; ++t) ka[t] = operand(t);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < OPS; ++t) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
          S[t % 4][nq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[t % RING], Q[nq][t / 4], S[t % 4][nq], 0, 0, 0);
        if (t + RING < OPS) ka[t % RING] = operand(t + RING);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    auto mask = [&](int t) {
      const int key0 = first_key + t * TILE;
      if (key0 + TILE - 1 > first_limit) {
#pragma unroll
        for (int kb = 0; kb < 4; ++kb)
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + 16 * kb + 4 * g4 + i > limit[nq]) S[kb][nq][i] = -INFINITY;
            // Four comparisons at a time: all 32 take 64 scalar registers, and those that every tile needs are spilled (a chunk of 2,048
            // tokens 945 instead of 918 us, 24 chunks of heads of 64 140 instead of 134).
            __builtin_amdgcn_sched_barrier(0);
          }
      }
    };
    auto row_max = [&](int nq) {
      float m = S[0][nq][0];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, S[kb][nq][i]);
      return quad_max(m);
    };
    auto reference = [&](int nq) { return mref[nq] == -INFINITY ? 0.f : mref[nq] * c_log2; };  // -inf: no key is seen
    // probabilities of block j = NQ kb + nq, rounded to bf16 for the product with V; their sum is taken before rounding
    auto slice = [&](int j, const float (&mc)[NQ], bf16x8 (&Pn)[2][NQ], float (&lacc)[NQ]) {
      const int kb = j / NQ, nq = j % NQ;
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const f32x2 pr = {__builtin_amdgcn_exp2f(__builtin_fmaf(S[kb][nq][e], c_log2, -mc[nq])),
                          __builtin_amdgcn_exp2f(__builtin_fmaf(S[kb][nq][e + 1], c_log2, -mc[nq]))};
        const bf16x2 pk = __builtin_convertvector(pr, bf16x2);
        lacc[nq] += pr[0] + pr[1];
        Pn[kb >> 1][nq][(kb & 1) * 4 + e] = pk[0];
        Pn[kb >> 1][nq][(kb & 1) * 4 + e + 1] = pk[1];
      }
    };
    auto accept = [&](const bf16x8 (&Pn)[2][NQ], const float (&lacc)[NQ]) {
      bool unsafe = false;
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        unsafe = unsafe || !(lacc[nq] <= SAFE_SUM);  // also NaN
        lsum[nq] += lacc[nq];
#pragma unroll
        for (int c32 = 0; c32 < 2; ++c32) Pb[c32][nq] = Pn[c32][nq];
      }
      bad = bad || __any(unsafe);
    };
    // O^T += V^T P^T for the tile in Pb, interleaved with the softmax of the tile in S
    auto product = [&](const unsigned char* vbuf, auto overlap_c, bf16x8 (&Pn)[2][NQ], float (&lacc)[NQ]) {
      constexpr int OPS = 2 * CB;
      float mc[NQ];
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) mc[nq] = reference(nq);
      auto operand = [&](int t) {
        const unsigned char* v = vbuf + (t / CB) * 32 * ROWB + vtr[t % CB];
        return lds_operand_tr(v, v + 16 * ROWB);
      };
      bf16x8 va[RING];
#pragma unroll
      for (int t = 0; t < RING; ++t) va[t] = operand(t);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < OPS; ++t) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
          O[t % CB][nq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[t % RING], Pb[t / CB][nq], O[t % CB][nq], 0, 0, 0);
        if (t + RING < OPS) va[t % RING] = operand(t + RING);
        if (decltype(overlap_c)::value) {
#pragma unroll
          for (int j = t * (4 * NQ) / OPS; j < (t + 1) * (4 * NQ) / OPS; ++j) slice(j, mc, Pn, lacc);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    };

    // Once; and, where some row's probabilities left the safe range, once more with the true maxima.
    for (int again = 0; tiles > 0; ++again) {
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        mref[nq] = -INFINITY;
        lsum[nq] = 0.f;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) O[cb][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      bad = false;
      if (again) {
        for (int t = 0; t < tiles; ++t) {
          issue_k(source(t, look_up(t)), 0);
          wait_loads<0>();
          __syncthreads();
          scores(smem);
          mask(t);
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) mref[nq] = fmaxf(mref[nq], row_max(nq));
          __syncthreads();
        }
      }
      Rows from = source(0, look_up(0));  // of the last tile whose K was issued
      issue_k(from, 0);
      auto issue_next = [&](int t, int page, int vbuf, int kbuf) {  // V of tile t - 1 and K of tile t
        issue_v(from, vbuf);
        from = source(t, page);
        issue_k(from, kbuf);
      };
#pragma unroll
      for (int t = 1; t <= AHEAD; ++t) issue_next(t, look_up(t), (t - 1) * TILE_BYTES, t * TILE_BYTES);
      int page = look_up(AHEAD + 1);
      wait_loads<AHEAD * 2 * LOADS>();  // K of tile 0
      barrier_with_loads();
      scores(smem);
      mask(0);
      {
        bf16x8 Pn[2][NQ];
        float lacc[NQ], mc[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
          if (!again) {
            mref[nq] = row_max(nq);
            bad = bad || __any(mref[nq] == -INFINITY);  // a row without a key in its first tile has no reference yet
          }
          mc[nq] = reference(nq);
          lacc[nq] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4 * NQ; ++j) slice(j, mc, Pn, lacc);
        accept(Pn, lacc);
      }
      wait_loads<(AHEAD - 1) * 2 * LOADS>();
      barrier_with_loads();
      // Step t: the scores of tile t, then the product of tile t - 1 and the softmax of tile t.  Tile t is in buffer t % BUFS; K of
      // tile t + AHEAD goes where K of tile t - 1 was, V of the tile before it where V of tile t - 2 was.
      int buf = 0;  // of tile t - 1
      auto after = [&](int b) { return b == AHEAD * TILE_BYTES ? 0 : b + TILE_BYTES; };
      auto next_tile = [&](int t, int old) {
        issue_next(t + AHEAD, page, old == 0 ? AHEAD * TILE_BYTES : old - TILE_BYTES, old);
        page = look_up(t + AHEAD + 1);
        wait_loads<(AHEAD - 1) * 2 * LOADS>();  // K of tile t + 1 and V of tile t
        barrier_with_loads();
      };
      int t = 1;
      if (idle) {
        for (; t < tiles; ++t, buf = after(buf)) next_tile(t, buf);
      }
      for (; t < tiles; ++t) {
        const int old = buf;
        buf = after(old);
        scores(smem + buf);
        mask(t);
        bf16x8 Pn[2][NQ];
        float lacc[NQ];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) lacc[nq] = 0.f;
        product(smem + VBUF + old, std::true_type{}, Pn, lacc);
        accept(Pn, lacc);
        next_tile(t, old);
      }
      {
        bf16x8 Pn[2][NQ];
        float lacc[NQ];
        product(smem + VBUF + buf, std::false_type{}, Pn, lacc);
      }
      wait_loads<0>();  // the empty ones too: the next loads go over their places
      if (again) break;
      if (lane == 0) gave_up[wave] = bad ? 1 : 0;
      __syncthreads();
      int any = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) any |= gave_up[w];
      if (__builtin_amdgcn_readfirstlane(any) == 0) break;
      __syncthreads();
    }
    if (lane == 0) wave_lost[wave] = first_lost;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) first_lost = wave_lost[w] < first_lost ? wave_lost[w] : first_lost;

#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = wave * ROWS_PER_WAVE + nq * 16 + l16;
      float l = tiles > 0 ? quad_sum(lsum[nq]) : 0.f;
      if (r >= block_rows) continue;
      if (limit[nq] >= first_lost) l = NAN;
      const float inv = l == 0.f ? 0.f : 1.f / l;  // 0: no key is seen
      const float lse = tiles > 0 ? mref[nq] * a.scale + __logf(l) : -INFINITY;
      const Place dst = walk.place(a, p, r);
      auto value = [&](int cb) { return tiles > 0 ? O[cb][nq] * inv : f32x4{0.f, 0.f, 0.f, 0.f}; };
      if (dst.partial) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) *reinterpret_cast<f32x4*>(static_cast<float*>(dst.row) + 16 * cb + 4 * g4) = value(cb);
      } else {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
          *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(dst.row) + 16 * cb + 4 * g4) = __builtin_convertvector(value(cb), bf16x4);
      }
      if (g4 == 0 && dst.lse) *dst.lse = lse;
    }
    walk.note_cut(a);
    __syncthreads();  // all reads of the tiles are over before the next block's loads come
  }
}

}  // namespace

int launch_paged_chunk(const PagedArgs& a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.D == 128) paged_chunk_kernel<128><<<a.groups, THREADS, 0, s>>>(a);
  else paged_chunk_kernel<64><<<a.groups, THREADS, 0, s>>>(a);
  return (int)hipGetLastError();
}

}  // namespace pa
