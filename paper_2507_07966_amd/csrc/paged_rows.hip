// Attention of new tokens over their pages for calls of few rows a sequence (single tokens, short chunks), and for fp32.
//   out_i = sum_j e^{s_ij - LSE_i} v_j,   s_ij = scale <q_i, k_j>,   j up to the token's own position.
//
// Bound: memory.  A token of r = Hq / Hkv rows a kv head does 4 r D operations on 4 D bytes of a key and its value (bf16), so a
// call runs at the rate at which keys and values come in.  Mapping:
//   - A workgroup takes shares of the line of paged_sched.h; a block is up to 16 NQ stacked rows (query heads of a GQA
//     group, and new tokens), which all use every key that is loaded.
//   - The 4 wavefronts split the KEYS of a tile, not the rows: a wavefront has its own 16 KiB stages in LDS, filled by direct-to-LDS
//     loads (STAGES of them in flight or in use: 128 KiB a compute unit), and there is no barrier inside a block.  The
//     kernel waits for the stage that it is about to read only, but the compiler, which knows of these loads and cannot tell the
//     ring's places apart, adds a wait for all of them before every second stage in all but the two instances of heads of 64 and 16
//     rows.  It also waits for them before the joint, which lies over the other wavefronts' rings.  A page is looked up once for 16 keys (page
//     sizes are multiples of 16), in scalar registers one stage ahead; the loads' range ends at the last key or is empty where a page
//     is missing, so LDS holds zeros there and nothing outside the cache is read.  A row that sees a key without a page, which is one whose
//     limit is not below the smallest such key, becomes NaN at the end.
//   - Scores are formed transposed, S^T = K Q^T, so that a lane holds scores of one query and the probabilities are the operand of
//     O^T += V^T P^T as they are.  bf16: v_mfma_f32_16x16x32_bf16, V read transposed from LDS (ds_read_b64_tr_b16).
//     fp32: v_mfma_f32_16x16x4_f32; channels are dealt to the steps of the product such that every LDS read is 16 bytes a
//     lane.
//   - Online softmax with the true running maximum a wavefront; the accumulators are rescaled only when some row's maximum moved.  At the
//     end of a block the wavefronts' results are joined through LDS.
//
// Measured (28 + 4 heads of 128, bf16): one token each of 64 sequences of 700 ... 17,000 keys, 1.08 GB of keys and values: 187 ... 193 us,
// 5.6 ... 5.8 TB/s (15.4 ms in a kernel without direct-to-LDS loads, MFMA and equal shares).  8 rollouts over one video of 32,768 keys:
// 27 us, of which 16 are its bytes; one sequence of 1,100 keys: 10.5 us: there latency counts, a chain of four reads to the
// first key and the joint at the end.  fp32, 5 chunks of 5 ... 106 tokens: 61 us, the matrix pipe busy 50 % of the cycles, 0.4
// LDS bank conflicts a cycle of LDS use.
// 8 wavefronts of one stage each instead of 4 of two: one token 16.5 (then 16.1) and fp32 83.6 us (72.9).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "common.h"
#include "mfma_tiles.h"
#include "paged.h"
#include "paged_device.h"

namespace pa {
namespace {

using namespace mt;

constexpr int WAVES = PAGED_ROWS_WAVES, THREADS = WAVES * 64, STAGES = 2;
constexpr int HALF_STAGE = PAGED_ROWS_HALF_STAGE;  // bytes of keys, and of values
constexpr int LOADS = 2 * HALF_STAGE / 1024;  // of a stage

// What differs between the data types: the operands of the two products.
template <int D, int NQ>
struct CoreBf16 {
  typedef __bf16 T;
  static constexpr int ROWB = 2 * D, KEYS = HALF_STAGE / ROWB, KB = KEYS / 16, KS = D / 32, CB = D / 16;
  bf16x8 Q[NQ][KS];
  f32x4 O[CB][NQ];
  int koff[KS], vtr[CB];
  __device__ static int swizzle(int row) { return swizzle16(row, ROWB); }
  // (the swizzle is an exclusive or on the chunk's bits, so the addresses of a lane differ by one, too)
  __device__ void init(int l16, int g4) {
    const int k0 = l16 * ROWB + ((g4 ^ swizzle(l16)) << 4), r = 4 * g4 + (l16 >> 2);
    const int v0 = r * ROWB + ((((l16 & 3) >> 1) ^ swizzle(r)) << 4) + (l16 & 1) * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = k0 ^ (ks << 6);
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) vtr[cb] = v0 ^ (cb << 5);
  }
  __device__ void load_q(int nq, const T* row, int g4) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      Q[nq][ks] = row ? *reinterpret_cast<const bf16x8*>(row + 32 * ks + 8 * g4) : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
  }
  // the operands of a stage; its place in LDS is free once they have arrived
  bf16x8 K[KB][KS], V[KB / 2][CB];
  __device__ void read(const unsigned char* kbuf, const unsigned char* vbuf) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) K[kb][ks] = lds_operand(kbuf + kb * 16 * ROWB + koff[ks]);
#pragma unroll
    for (int c32 = 0; c32 < KB / 2; ++c32)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const unsigned char* p = vbuf + c32 * 32 * ROWB + vtr[cb];
        V[c32][cb] = lds_operand_tr(p, p + 16 * ROWB);
      }
  }
  __device__ void scores(f32x4 (&S)[KB][NQ]) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) S[kb][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) S[kb][nq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(K[kb][ks], Q[nq][ks], S[kb][nq], 0, 0, 0);
  }
  // P holds the probabilities of the stage in the layout of S; rounded to bf16, as everywhere in this library, for the product with V
  __device__ void accumulate(const f32x4 (&P)[KB][NQ]) {
#pragma unroll
    for (int c32 = 0; c32 < KB / 2; ++c32) {
      bf16x8 pb[NQ];
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        const bf16x4 lo = __builtin_convertvector(P[2 * c32][nq], bf16x4), hi = __builtin_convertvector(P[2 * c32 + 1][nq], bf16x4);
        pb[nq] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) O[cb][nq] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(V[c32][cb], pb[nq], O[cb][nq], 0, 0, 0);
    }
  }
  // this lane's channels of query column nq, times f, into its row
  __device__ void store(f32x4* row, int nq, float f, int g4, int l16) const {
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) row[(g4 ^ l16) ^ (4 * cb)] = O[cb][nq] * f;
  }
};

template <int D, int NQ>
struct CoreF32 {
  typedef float T;
  static constexpr int ROWB = 4 * D, KEYS = HALF_STAGE / ROWB, KB = KEYS / 16, KS = D / 16, CB = D / 16;
  f32x4 Q[NQ][KS];  // step 4 s + e of the product contracts channels g4 D / 4 + 4 s + e
  f32x4 O[CB][NQ];  // register i of block 4 b + e is channel 64 b + 4 (4 g4 + i) + e
  int koff[KS], voff[4];
  __device__ static int swizzle(int row) { return row & 15; }
  __device__ void init(int l16, int g4) {
    const int k0 = l16 * ROWB + (((g4 * KS) ^ swizzle(l16)) << 4);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) koff[ks] = k0 ^ (ks << 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) voff[i] = (4 * g4 + i) * ROWB + ((l16 ^ swizzle(4 * g4 + i)) << 4);
  }
  __device__ void load_q(int nq, const T* row, int g4) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      Q[nq][ks] = row ? *reinterpret_cast<const f32x4*>(row + g4 * (D / 4) + 4 * ks) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  f32x4 K[KB][KS], V[KB][4][D / 64];
  __device__ void read(const unsigned char* kbuf, const unsigned char* vbuf) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) K[kb][ks] = *reinterpret_cast<const f32x4*>(kbuf + kb * 16 * ROWB + koff[ks]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < D / 64; ++b) V[kb][i][b] = *reinterpret_cast<const f32x4*>(vbuf + kb * 16 * ROWB + voff[i] + b * 256);
    }
  }
  __device__ void scores(f32x4 (&S)[KB][NQ]) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) S[kb][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) S[kb][nq] = __builtin_amdgcn_mfma_f32_16x16x4f32(K[kb][ks][e], Q[nq][ks][e], S[kb][nq], 0, 0, 0);
  }
  __device__ void accumulate(const f32x4 (&P)[KB][NQ]) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i)  // contraction slot g4 of this step is key 4 g4 + i
#pragma unroll
        for (int b = 0; b < D / 64; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int nq = 0; nq < NQ; ++nq)
              O[4 * b + e][nq] = __builtin_amdgcn_mfma_f32_16x16x4f32(V[kb][i][b][e], P[kb][nq][i], O[4 * b + e][nq], 0, 0, 0);
  }
  __device__ void store(f32x4* row, int nq, float f, int g4, int l16) const {
#pragma unroll
    for (int b = 0; b < D / 64; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 x = {O[4 * b][nq][i], O[4 * b + 1][nq][i], O[4 * b + 2][nq][i], O[4 * b + 3][nq][i]};
        row[(16 * b + 4 * g4 + i) ^ l16] = x * f;
      }
  }
};

template <template <int, int> class CoreT, int D, int NQ>
__global__ __launch_bounds__(THREADS, 1) void paged_rows_kernel(const PagedArgs a) {
  using Core = CoreT<D, NQ>;
  using T = typename Core::T;
  constexpr int KEYS = Core::KEYS, KB = Core::KB, ROWB = Core::ROWB, CB = Core::CB, ROWS = 16 * NQ;
  constexpr int GROUP_LOADS = 16 * ROWB / 1024;  // 1 KiB loads of 16 keys
  constexpr int LANES_PER_ROW = ROWB / 16, ROWS_PER_LOAD = 1024 / ROWB;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[WAVES * STAGES * 2 * HALF_STAGE];
  __shared__ float wave_max[WAVES][ROWS], wave_sum[WAVES][ROWS], row_scale[ROWS];
  constexpr int VECS = D / 4;  // 16-byte pieces of a row of fp32
  static_assert(WAVES * ROWS * D * 4 <= (int)sizeof(ring), "the joint fits the ring");

  Walk walk;
  if (!begin_walk<THREADS>(a, walk)) return;
  const PagedShape& shape = walk.shape;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const float c_log2 = a.scale * 1.4426950408889634f;

  Core core;
  core.init(l16, g4);
  unsigned loff[GROUP_LOADS];  // byte offset of this lane's 16 bytes in 16 rows of the cache, for each load of them
#pragma unroll
  for (int n = 0; n < GROUP_LOADS; ++n) {
    const int row = n * ROWS_PER_LOAD + lane / LANES_PER_ROW;
    loff[n] = (unsigned)(row * ROWB + (((lane % LANES_PER_ROW) ^ Core::swizzle(row)) << 4));
  }
  unsigned char* const my_ring = ring + wave * (STAGES * 2 * HALF_STAGE);

  for (; walk.more(); walk.next(a)) {
    const Piece p = walk.piece();
    const Segment& seg = walk.seg;
    const int block_rows = walk.block.rows;
    const int32_t* const table = a.page_table + (int64_t)walk.table_row * a.table_width;
    const int first_key = seg.key0 + (p.tile0 << shape.tile_shift);
    const int last_key = (p.tile1 << shape.tile_shift) + seg.key0 < p.key_end ? (p.tile1 << shape.tile_shift) + seg.key0 : p.key_end;
    // stages of this wavefront: stage s covers keys first_key + (WAVES s + wave) KEYS ..
    const int span = last_key - first_key - wave * KEYS;
    const int stages = span > 0 ? (span + WAVES * KEYS - 1) / (WAVES * KEYS) : 0;
    const int key_base = first_key + wave * KEYS;

    const uint32_t page_bytes = ((uint32_t)shape.Hkv << a.page_shift) * (uint32_t)ROWB;
    const int64_t head_bytes = ((int64_t)walk.head << a.page_shift) * ROWB;
    int first_lost = last_key > shape.capacity ? shape.capacity : 0x7fffffff;  // smallest key without a page: rows that see it become NaN
    const int end = last_key < shape.capacity ? last_key : shape.capacity;
    int pid[KB];  // pages of the next stage to be loaded
    auto look_up = [&](int s) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) pid[kb] = page_of(a, table, key_base + s * WAVES * KEYS + 16 * kb);
    };
    using B0 = std::integral_constant<int, 0>;
    using B1 = std::integral_constant<int, 1>;
    auto load = [&](int s, auto buf_c) {
      unsigned char* const dst = my_ring + decltype(buf_c)::value * 2 * HALF_STAGE;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const Rows from = find_rows(a, pid[kb], page_bytes, head_bytes, key_base + s * WAVES * KEYS + 16 * kb, end, 16, ROWB, first_lost);
        const rsrc_t kr = rows_rsrc(a.k_cache, from), vr = rows_rsrc(a.v_cache, from);
#pragma unroll
        for (int n = 0; n < GROUP_LOADS; ++n) load_chunk_to_lds(kr, dst + kb * 16 * ROWB + n * 1024, loff[n], 0);
#pragma unroll
        for (int n = 0; n < GROUP_LOADS; ++n) load_chunk_to_lds(vr, dst + HALF_STAGE + kb * 16 * ROWB + n * 1024, loff[n], 0);
      }
    };

    look_up(0);
    int limit[NQ];  // last key that query column nq sees
    int least = 0x7fffffff;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = nq * 16 + l16;
      const T* row = nullptr;
      limit[nq] = 0x7fffffff;
      if (r < block_rows) {
        const int tok = walk.row_token(r);
        row = static_cast<const T*>(a.q) + (int64_t)(seg.token0 + tok) * a.q_stride + walk.row_head(r, tok) * D;
        limit[nq] = walk.shared ? p.key_end - 1 : row_limit(shape, seg, tok);
      }
      core.load_q(nq, row, g4);
      least = limit[nq] < least ? limit[nq] : least;
    }
    load(0, B0{});  // empty where this wavefront has no stage: the compiler counts what is under way behind the queries
    if (stages > 1) {
      look_up(1);
      load(1, B1{});
      if (stages > 2) look_up(2);
    }
#pragma unroll
    for (int x = 1; x < 16; x *= 2) {
      const int other = __shfl_xor(least, x);
      least = other < least ? other : least;
    }
    const int first_limit = __builtin_amdgcn_readfirstlane(least);  // keys up to this one are seen by every row

    float top[NQ], sum[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      top[nq] = -INFINITY;
      sum[nq] = 0.f;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) core.O[cb][nq] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    auto compute = [&](int s) {
      f32x4 S[KB][NQ];
      core.scores(S);
      const int key0 = key_base + s * WAVES * KEYS;
      const int seen = first_limit < last_key - 1 ? first_limit : last_key - 1;
      if (key0 + KEYS - 1 > seen) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int nq = 0; nq < NQ; ++nq) {
            const int last = limit[nq] < last_key - 1 ? limit[nq] : last_key - 1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = key0 + 16 * kb + 4 * g4 + i;
              if (key > last) S[kb][nq][i] = -INFINITY;
            }
          }
      }
      float alpha[NQ];
      bool moved = false;
#pragma unroll
      for (int nq = 0; nq < NQ; ++nq) {
        float t = S[0][nq][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) t = fmaxf(t, S[kb][nq][i]);
        t = quad_max(t);
        const float next = fmaxf(top[nq], t);
        alpha[nq] = next == top[nq] ? 1.f : __builtin_amdgcn_exp2f((top[nq] - next) * c_log2);
        moved = moved || next != top[nq];
        top[nq] = next;
        const float ref = next == -INFINITY ? 0.f : next * c_log2;
        float part = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            S[kb][nq][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[kb][nq][i], c_log2, -ref));
            part += S[kb][nq][i];
          }
        sum[nq] = sum[nq] * alpha[nq] + part;
      }
      if (__any(moved)) {
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) core.O[cb][nq] *= alpha[nq];
      }
      core.accumulate(S);
    };
    auto step = [&](int s, auto buf_c) {
      constexpr int BUF = decltype(buf_c)::value;
      const unsigned char* const kbuf = my_ring + BUF * 2 * HALF_STAGE;
      // this stage's loads are done when at most those of the next one are under way
      if (s + 1 < stages) wait_loads<LOADS>(); else wait_loads<0>();
      core.read(kbuf, kbuf + HALF_STAGE);
      if (s + 2 < stages) {  // all operands are in registers: the loads of the stage after the next one go over them
        wait_lds_reads();
        load(s + 2, buf_c);
        if (s + 3 < stages) look_up(s + 3);
      }
      compute(s);
    };
    for (int s = 0; s < stages; s += 2) {
      step(s, B0{});
      if (s + 1 < stages) step(s + 1, B1{});
    }

    // ---- join the wavefronts: reference maxima, then the outputs, all of the block's rows at once through LDS (16-byte chunk c of row r
    //      at chunk c ^ (r & 15): rows written by 16 lanes at one chunk fall on all banks)
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const float l = limit[nq] >= first_lost ? NAN : quad_sum(sum[nq]);
      if (g4 == 0) {
        wave_max[wave][nq * 16 + l16] = top[nq];
        wave_sum[wave][nq * 16 + l16] = l;
      }
    }
    __syncthreads();  // all loads are done and all reads of the ring are over
    f32x4* const joint = reinterpret_cast<f32x4*>(ring);
    auto factor = [&](float from, float to) { return from == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((from - to) * c_log2); };
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
      const int r = nq * 16 + l16;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) m = fmaxf(m, wave_max[w][r]);
      if (r < block_rows) core.store(joint + (wave * ROWS + r) * VECS, nq, factor(top[nq], m), g4, l16);
    }
    if (tid < block_rows) {
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) m = fmaxf(m, wave_max[w][tid]);
#pragma unroll
      for (int w = 0; w < WAVES; ++w) l += wave_sum[w][tid] * factor(wave_max[w][tid], m);
      row_scale[tid] = l == 0.f ? 0.f : 1.f / l;  // 0: no key is seen
      const Place dst = walk.place(a, p, tid);
      if (dst.lse) *dst.lse = m * a.scale + __logf(l);
    }
    __syncthreads();
    for (int idx = tid; idx < block_rows * VECS; idx += THREADS) {
      const int r = idx / VECS, v = idx % VECS;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) o += joint[(w * ROWS + r) * VECS + (v ^ (r & 15))];
      write_row<T>(walk.place(a, p, r), 4 * v, o * row_scale[r]);
    }
    walk.note_cut(a);
    __syncthreads();  // the joint is read before the next block's loads come
  }
}

}  // namespace

int launch_paged_rows(const PagedArgs& a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
#define PA_ROWS(CORE, DD, NQ) paged_rows_kernel<CORE, DD, NQ><<<a.groups, THREADS, 0, s>>>(a)
#define PA_ROWS_D(CORE, NQ) \
  if (a.D == 128) PA_ROWS(CORE, 128, NQ); else PA_ROWS(CORE, 64, NQ)
  if (a.dtype == PA_BF16) {
    if (a.blocks16 == 1) { PA_ROWS_D(CoreBf16, 1); }
    else if (a.blocks16 == 2) { PA_ROWS_D(CoreBf16, 2); }
    else { PA_ROWS_D(CoreBf16, 4); }
  } else {
    if (a.blocks16 == 1) { PA_ROWS_D(CoreF32, 1); } else { PA_ROWS_D(CoreF32, 2); }
  }
#undef PA_ROWS_D
#undef PA_ROWS
  return (int)hipGetLastError();
}

}  // namespace pa
