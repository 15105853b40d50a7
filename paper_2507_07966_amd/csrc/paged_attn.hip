// Attention of each sequence's new tokens over its pages: out_i = sum_j e^{s_ij - LSE_i} v_j over the keys j up to the
// token's own position, with s_ij = scale <q_i, k_j>.
//
// One workgroup per (token, kv head); each wavefront takes rows of the group in turn, a lane per key for the scores and
// a lane per channel for the values, with the running maximum and sum of the softmax.
#include <hip/hip_runtime.h>

#include "common.h"
#include "paged.h"

namespace pa {
namespace {

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_attn_kernel(const PagedArgs a) {
  const int t = blockIdx.x, c = blockIdx.y;
  __shared__ int seq;
  __shared__ float qs[4][D];
  if (threadIdx.x == 0) seq = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.B; b += 256)
    if (a.cu_new[b] <= t && t < a.cu_new[b + 1]) seq = b;
  __syncthreads();
  const int b = seq;
  if (b < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t cap = (int64_t)a.table_width << a.page_shift;
  const int64_t pos = (int64_t)a.seq_lens[b] - a.cu_new[b + 1] + t;
  const int64_t keys = pos + 1 < 0 ? 0 : pos + 1 > cap + 1 ? cap + 1 : pos + 1;  // one past the table: a key without a page
  for (int j = wave; j < a.group; j += 4) {
    const int h = c * a.group + j;
    const T* q = static_cast<const T*>(a.q) + t * a.q_stride + (int64_t)h * D;
    for (int e = lane; e < D; e += 64) qs[wave][e] = (float)q[e];
    float m = -INFINITY, l = 0.f, acc[D / 64] = {};
    for (int64_t k0 = 0; k0 < keys; k0 += 64) {
      const int64_t key = k0 + lane;
      float s = -INFINITY;
      int64_t row = -1;
      if (key < keys) {
        const int64_t idx = key >> a.page_shift;
        const int64_t page = idx < a.table_width ? a.page_table[(int64_t)b * a.table_width + idx] : -1;
        s = NAN;
        if (page >= 0 && page < a.num_pages) {
          row = (((page * a.Hkv + c) << a.page_shift) + (key & (((int64_t)1 << a.page_shift) - 1))) * D;
          const T* k = static_cast<const T*>(a.k_cache) + row;
          s = 0.f;
          for (int e = 0; e < D; ++e) s += qs[wave][e] * (float)k[e];
          s *= a.scale;
        }
      }
      float top = s;
      for (int x = 32; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
      const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
      const float p = expf(s - ref), alpha = expf(m - ref);
      float sum = p;
      for (int x = 32; x; x >>= 1) sum += __shfl_xor(sum, x);
      l = l * alpha + sum;
      m = mn;
      for (int e = 0; e < D / 64; ++e) acc[e] *= alpha;
      for (int i = 0; i < 64; ++i) {
        const int64_t r = __shfl(row, i);
        const float w = __shfl(p, i);
        if (r >= 0)
          for (int e = 0; e < D / 64; ++e) acc[e] += w * (float)static_cast<const T*>(a.v_cache)[r + e * 64 + lane];
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;  // 0: no key is visible
    for (int e = 0; e < D / 64; ++e)
      static_cast<T*>(a.out)[((int64_t)t * a.Hq + h) * D + e * 64 + lane] = (T)(acc[e] * inv);
    if (a.lse && lane == 0) a.lse[(int64_t)h * a.T + t] = m + logf(l);
  }
}

}  // namespace

int launch_paged_attn(const PagedArgs& a, void* stream) {
  const dim3 grid((unsigned)a.T, (unsigned)a.Hkv);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.dtype == PA_BF16) {
    if (a.D == 128) paged_attn_kernel<__bf16, 128><<<grid, 256, 0, s>>>(a);
    else paged_attn_kernel<__bf16, 64><<<grid, 256, 0, s>>>(a);
  } else {
    if (a.D == 128) paged_attn_kernel<float, 128><<<grid, 256, 0, s>>>(a);
    else paged_attn_kernel<float, 64><<<grid, 256, 0, s>>>(a);
  }
  return (int)hipGetLastError();
}

}  // namespace pa
