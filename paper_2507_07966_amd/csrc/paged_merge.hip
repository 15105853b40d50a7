// Joins the pieces of blocks whose keys were cut: LSE = ln sum_i e^{LSE_i}, out = sum_i e^{LSE_i - LSE} O_i.
//
// Without shared keys, workgroup (share, y) looks whether its share begins a block that it does not end, and merges rows of that block: the
// last piece that share left and what the shares after it left of the same block.  With shared keys every row has
// pieces of its own keys and of the shared ones: a workgroup per row finds both from the line.  Bound: latency.  A row's D / 4 vectors are
// spread over lanes; the groups of lanes that a workgroup has for it are split between rows and pieces, by how many pieces a row has, and
// the sums of a row's groups are joined through LDS.  Measured: one token of 28 heads over 1,100 keys, cut into a few pieces, 3.4 us; 8 rollouts over
// a shared video, whose 224 rows have up to 64 pieces each, 5.8 us; a chunk of 2,048 tokens, whose blocks are cut twice, 16 us.
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

template <int D>
struct Joint {
  static constexpr int VECS = D / 4, GROUPS = THREADS / VECS;  // lanes of a row, groups of them in a workgroup
  f32x4 acc[GROUPS][VECS];
  float top[GROUPS], sum[GROUPS];
};

// This lane's vector of a row of one or two lists of pieces, STEP of which it has in flight, `parts` groups of lanes (a power of
// two, in a row) to a row.  Every thread of the workgroup calls it; `live`: the row exists.
template <typename T, int D, int STEP>
__device__ inline void merge_row(const PagedArgs& a, const Pieces (&list)[2], int lists, int parts, bool live, int64_t t, int64_t h,
                                 Joint<D>& joint) {
  using J = Joint<D>;
  const int vec = threadIdx.x % J::VECS, group = threadIdx.x / J::VECS, part = group & (parts - 1);
  const int block_rows = a.shape.block_rows;
  const int n0 = list[0].count, n = !live ? 0 : n0 + (lists > 1 ? list[1].count : 0);
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
  for (int i0 = part; i0 < n; i0 += parts * STEP) {
    float l[STEP];
    f32x4 o[STEP];
#pragma unroll
    for (int e = 0; e < STEP; ++e) {
      const int i = i0 + e * parts;
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
  if (parts > 1) {
    joint.acc[group][vec] = acc;
    if (vec == 0) {
      joint.top[group] = top;
      joint.sum[group] = sum;
    }
    __syncthreads();
    if (part) return;
    top = -INFINITY;
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) top = fmaxf(top, joint.top[group + p]);
    const float ref = top == -INFINITY ? 0.f : top;
    for (int p = 0; p < parts; ++p) {
      const float w = expf(joint.top[group + p] - ref);
      sum += w * joint.sum[group + p];
      acc += w * joint.acc[group + p][vec];
    }
  }
  if (!live) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;  // 0: no piece has a key that the row sees
  write_row<T>(Place{static_cast<T*>(a.out) + (t * a.Hq + h) * D, nullptr, false}, 4 * vec, acc * inv);
  if (vec == 0 && a.lse) a.lse[h * a.shape.T + t] = (top == -INFINITY ? 0.f : top) + logf(sum);
}

// Groups of lanes to a row of `pieces` pieces: a lane has STEP = 4 of them in flight, and should not need a second round.
template <int D>
__device__ inline int parts_for(int pieces) {
  int parts = 1;
  while (parts < Joint<D>::GROUPS && pieces > 4 * parts) parts *= 2;
  return parts;
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void merge_cuts_kernel(const PagedArgs a) {
  const int position = blockIdx.x;
  const int active = a.line->active;
  const PagedCut c = a.cuts[position];
  if (position >= active || c.tokens == 0) return;
  using J = Joint<D>;
  __shared__ J joint;
  const int pieces = c.last - c.first + 1, parts = parts_for<D>(pieces), rows = J::GROUPS / parts;  // rows of the workgroup
  const int left = c.tokens * a.shape.group - c.block * a.shape.block_rows;
  const int end = left < a.shape.block_rows ? left : a.shape.block_rows;
  for (int r0 = blockIdx.y * rows; r0 < end; r0 += gridDim.y * rows) {
    const int r = r0 + threadIdx.x / J::VECS / parts;
    const int m = c.block * a.shape.block_rows + r, i = (uint32_t)m / (uint32_t)a.shape.group, j = m - i * a.shape.group;
    const Pieces list[2] = {{pieces, (2 * (int64_t)c.first + 1) * a.shape.block_rows + r, false, c.first, r}, {}};
    merge_row<T, D, 4>(a, list, 1, parts, r < end, c.token0 + i, (int64_t)c.head * a.shape.group + j, joint);
    if (parts > 1) __syncthreads();
  }
}

template <typename T, int D>
__global__ __launch_bounds__(THREADS) void merge_rows_kernel(const PagedArgs a) {
  __shared__ Joint<D> joint;
  __shared__ int seq, own_start;
  __shared__ Lengths own_lengths;
  const int64_t t = blockIdx.x;
  const int64_t h = blockIdx.y;
  const PagedLine line = *a.line;
  const int32_t all_start = a.seg_start[0];
  const Lengths all_lengths = read_lengths(a, 0);
  if (threadIdx.x == 0) seq = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.shape.B; b += THREADS) {
    const Lengths l = read_lengths(a, b + 1);
    const int32_t start = a.seg_start[b + 1];
    if (l.cu0 <= t && t < l.cu1) {
      seq = b;
      own_lengths = l;
      own_start = start;
    }
  }
  __syncthreads();
  const int b = __builtin_amdgcn_readfirstlane(seq);
  if (b < 0 || line.active == 0) return;
  PagedShape s = a.shape;
  s.shared = line.shared;
  const int32_t share = line.share;
  const int head = (int)h / s.group, j = (int)h - head * s.group;
  auto pieces = [&](const Segment& g, int32_t start, bool shared) {
    const uint32_t m = (uint32_t)(t - g.token0) * s.group + j;
    const int block = (int)(m / (uint32_t)s.block_rows), r = (int)(m - (uint32_t)block * s.block_rows);
    const int32_t head_start = start + head * g.cost, c0 = head_start + blocks_cost(s, g, block), c1 = head_start + blocks_cost(s, g, block + 1);
    const int32_t first = div_small(c0, share), last = div_small(c1 - 1, share);
    if (first == last) return Pieces{1, ((shared ? (int64_t)s.T : 0) + t) * a.Hq + h, true, first, r};
    return Pieces{last - first + 1, (2 * (int64_t)first + 1) * s.block_rows + r, false, first, r};
  };
  const Segment own = segment_of(a, s, b + 1, own_lengths), all = segment_of(a, s, 0, all_lengths);
  const Pieces list[2] = {pieces(own, own_start, false), t < all.tokens ? pieces(all, all_start, true) : Pieces{}};
  merge_row<T, D, 8>(a, list, 2, Joint<D>::GROUPS, true, t, h, joint);
}

template <typename T, int D>
int launch(const PagedArgs& a, hipStream_t s) {
  if (a.shared_len) {
    merge_rows_kernel<T, D><<<dim3((unsigned)a.shape.T, (unsigned)a.Hq), THREADS, 0, s>>>(a);
  } else {
    // A block's rows are dealt to up to 16 workgroups: all rows of short blocks at once where they have many pieces
    const int64_t rows = (int64_t)a.shape.T * a.shape.group;  // of a kv head, in all
    const int most = rows < a.shape.block_rows ? (int)rows : a.shape.block_rows;
    merge_cuts_kernel<T, D><<<dim3((unsigned)a.groups, (unsigned)(most < 16 ? most : 16)), THREADS, 0, s>>>(a);
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
