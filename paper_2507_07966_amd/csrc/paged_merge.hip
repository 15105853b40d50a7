// Joins the pieces of blocks whose keys were cut: LSE = ln sum_i e^{LSE_i}, out = sum_i e^{LSE_i - LSE} O_i.
//
// Without shared keys, workgroup (share, y) looks whether its share begins a block that it does not end, and merges rows of that block: the
// last piece that share left and what the shares after it left of the same block.  With shared keys every row has
// pieces of its own keys and of the shared ones: a workgroup per row finds both from the line.  Bound: latency; a row's D / 4 vectors are
// spread over lanes and its pieces over groups of lanes, whose sums are joined through LDS.  Blocks of many rows have few pieces: there a
// workgroup takes several rows at once, a lane all pieces of its vector.
#include <hip/hip_runtime.h>

#include "paged.h"
#include "paged_device.h"

namespace pa {
namespace {

using namespace mt;

constexpr int THREADS = 256;

// The pieces of a row: `first` says where piece 0 is, piece i > 0 is what share first_share + i continued.
struct Pieces {
  int32_t count;
  int64_t row0;            // of piece 0: in `rows` if whole, else in the slots
  bool whole;
  int32_t first_share, row;  // further pieces: slot 2 (first_share + i), row `row` of it
};

template <int D, int PARTS_>
struct Joint {
  static constexpr int VECS = D / 4, PARTS = PARTS_;  // lanes of a row, pieces worked on at once
  static constexpr int ROWS = THREADS / VECS / PARTS;  // rows of a workgroup
  static_assert(PARTS == 1 || ROWS == 1, "either several pieces at once or several rows");
  f32x4 acc[PARTS][VECS];
  float top[PARTS], sum[PARTS];
};

// The row is made up of one or two lists of pieces.  With several pieces at once every thread of the workgroup calls it, for one row.
template <typename T, int D, int PARTS>
__device__ inline void merge_row(const PagedArgs& a, const Pieces (&list)[2], int lists, int64_t t, int64_t h, Joint<D, PARTS>& joint) {
  using J = Joint<D, PARTS>;
  const int vec = threadIdx.x % J::VECS, part = PARTS == 1 ? 0 : threadIdx.x / J::VECS;
  const int block_rows = a.shape.block_rows;
  const int n0 = list[0].count, n = n0 + (lists > 1 ? list[1].count : 0);
  auto at = [&](int i, const float*& o, const float*& l) {
    const Pieces& p = i < n0 ? list[0] : list[1];
    const int k = i < n0 ? i : i - n0;
    const int64_t row = k == 0 ? p.row0 : 2 * (int64_t)(p.first_share + k) * block_rows + p.row;
    const bool rows = k == 0 && p.whole;
    o = (rows ? a.rows : a.slots) + row * D + 4 * vec;
    l = (rows ? a.rows_lse : a.slot_lse) + row;
  };
  float top = -INFINITY, sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  constexpr int STEP = 4;  // pieces in flight a lane
  for (int i0 = part; i0 < n; i0 += J::PARTS * STEP) {
    float l[STEP];
    f32x4 o[STEP];
#pragma unroll
    for (int e = 0; e < STEP; ++e) {
      const int i = i0 + e * J::PARTS;
      l[e] = -INFINITY;
      o[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i < n) {
        const float *op, *lp;
        at(i, op, lp);
        l[e] = *lp;
        o[e] = *reinterpret_cast<const f32x4*>(op);
      }
    }
    float next = top;
#pragma unroll
    for (int e = 0; e < STEP; ++e) next = fmaxf(next, l[e]);
    const float ref = next == -INFINITY ? 0.f : next, alpha = expf(top - ref);
    acc *= alpha;
    sum *= alpha;
    top = next;
#pragma unroll
    for (int e = 0; e < STEP; ++e) {
      const float w = expf(l[e] - ref);  // NaN where the piece is
      sum += w;
      acc += w * o[e];
    }
  }
  if constexpr (PARTS > 1) {
    joint.acc[part][vec] = acc;
    if (vec == 0) {
      joint.top[part] = top;
      joint.sum[part] = sum;
    }
    __syncthreads();
    if (part) return;
    top = -INFINITY;
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) top = fmaxf(top, joint.top[p]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const float w = expf(joint.top[p] - ref);
      sum += w * joint.sum[p];
      acc += w * joint.acc[p][vec];
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;  // 0: no piece has a key that the row sees
  write_row<T>(Place{static_cast<T*>(a.out) + (t * a.Hq + h) * D, nullptr, false}, 4 * vec, acc * inv);
  if (vec == 0 && a.lse) a.lse[h * a.shape.T + t] = (top == -INFINITY ? 0.f : top) + logf(sum);
}

// blockIdx.y: which rows of the block
template <typename T, int D, int PARTS>
__global__ __launch_bounds__(THREADS) void merge_cuts_kernel(const PagedArgs a) {
  const int position = blockIdx.x;
  if (position >= a.line->active) return;
  const PagedCut c = a.cuts[position];
  if (c.tokens == 0) return;
  using J = Joint<D, PARTS>;
  __shared__ J joint;
  const int r = blockIdx.y * J::ROWS + (PARTS == 1 ? threadIdx.x / J::VECS : 0);
  const int m = c.block * a.shape.block_rows + r;
  if (m >= c.tokens * a.shape.group) return;
  const int i = (uint32_t)m / (uint32_t)a.shape.group, j = m - i * a.shape.group;
  const Pieces list[2] = {{c.last - c.first + 1, (2 * (int64_t)c.first + 1) * a.shape.block_rows + r, false, c.first, r}, {}};
  merge_row<T, D, PARTS>(a, list, 1, c.token0 + i, (int64_t)c.head * a.shape.group + j, joint);
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void merge_rows_kernel(const PagedArgs a) {
  constexpr int PARTS = THREADS / (D / 4);
  __shared__ Joint<D, PARTS> joint;
  __shared__ int seq;
  const int64_t t = blockIdx.x;
  const int64_t h = blockIdx.y;
  if (a.line->active == 0) return;
  if (threadIdx.x == 0) seq = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.shape.B; b += THREADS)
    if (a.cu_new[b] <= t && t < a.cu_new[b + 1]) seq = b;
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(seq);
  if (b < 0) return;
  PagedShape s = a.shape;
  s.shared = a.line->shared;
  const int32_t share = a.line->share;
  const int head = (int)h / s.group, j = (int)h - head * s.group;
  auto pieces = [&](const Segment& g, int32_t start, bool shared) {
    const uint32_t m = (uint32_t)(t - g.token0) * s.group + j;
    const int block = (int)(m / (uint32_t)s.block_rows), r = (int)(m - (uint32_t)block * s.block_rows);
    const int32_t c0 = start + head * g.cost + blocks_cost(g, block), c1 = c0 + g.first_cost + block * g.more_cost;
    const int32_t first = div_small(c0, share), last = div_small(c1 - 1, share);
    if (first == last) return Pieces{1, ((shared ? (int64_t)s.T : 0) + t) * a.Hq + h, true, first, r};
    return Pieces{last - first + 1, (2 * (int64_t)first + 1) * s.block_rows + r, false, first, r};
  };
  const Segment own = load_segment(a, s, b + 1), all = load_segment(a, s, 0);
  const Pieces list[2] = {pieces(own, a.seg_start[b + 1], false), t < all.tokens ? pieces(all, a.seg_start[0], true) : Pieces{}};
  merge_row<T, D, PARTS>(a, list, 2, t, h, joint);
}

template <typename T, int D>
int launch(const PagedArgs& a, hipStream_t s) {
  if (a.shared_len) {
    merge_rows_kernel<T, D><<<dim3((unsigned)a.shape.T, (unsigned)a.Hq), THREADS, 0, s>>>(a);
  } else {
    const int64_t rows = (int64_t)a.shape.T * a.shape.group;  // of a kv head, in all
    const int most = rows < a.shape.block_rows ? (int)rows : a.shape.block_rows;
    constexpr int LANES = THREADS / (D / 4);
    if (a.shape.block_rows > 64) merge_cuts_kernel<T, D, 1><<<dim3((unsigned)a.groups, (unsigned)((most + LANES - 1) / LANES)), THREADS, 0, s>>>(a);
    else merge_cuts_kernel<T, D, LANES><<<dim3((unsigned)a.groups, (unsigned)most), THREADS, 0, s>>>(a);
  }
  return (int)hipGetLastError();
}

}  // namespace

int launch_paged_merge(const PagedArgs& a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.dtype == PA_BF16) return a.D == 128 ? launch<__bf16, 128>(a, s) : launch<__bf16, 64>(a, s);
  return a.D == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace pa
