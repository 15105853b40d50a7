// Rotary positions with several axes, and the append of new keys and values to a paged cache.
//
// Pair i of token t is turned by a = positions[axis(i)][t] * inv_freq[i]; the gradient is the turn by -a.  Bound: memory (every
// element is read and written once: 4 bytes an element in bf16 for 3 operations).
//
// Mapping: a head's channels are split into units of W channel pairs (16 bytes of each of the two channels of a pair, or of W / 2
// neighbouring pairs), of W channels that pass through, and of single pairs and channels where a size is no multiple of W.
// A thread owns one unit of one token, forms the unit's sines and cosines once in registers, and turns that unit of HPT heads: four or
// eight in large calls, two in small ones, where latency counts.  The heads' loads are issued before the sines are worked out
// (32,768 tokens, 28 + 4 heads of 128, bf16: 132 -> 109 us, 4.9 TB/s).  The largest calls store past the caches (139 -> 132 us before that;
// appended chunks, whose values are only copied, 50 -> 37 us).  Vector accesses are declared with the alignment of an element, so slices at any offset take the same path.
#include <hip/hip_runtime.h>

#include "common.h"
#include "paged.h"

namespace pa {
namespace {

constexpr int THREADS = 256;

// cos and sin of `pos * inv_freq`.  A turn of 2^31 radians rounded to 53 bits is off by 4 units of fp32, so the frequency in quarter turns is held
// as a number of 64 bits and the fp32 rest that these leave, and the whole quarter turns go off inside the product's fma.  What is left is off by one
// fp32 rounding (angles up to 2^51 radians), |x| <= pi / 4, and goes through the Taylor series, whose first left-out terms are x^11 / 11! of the
// sine (relative 2e-9) and x^12 / 12! of the cosine.  The worst of 12,000 angles up to 2^41 radians: 1.8 units of 2^-24 (31 at
// 2^33 and 8,111 at 2^41 radians without the rest).
// (The rest in fp32 also saves registers: with 82 scalar ones instead of 80 only 7 wavefronts fit a SIMD, and fp32 gradients of 5,377 tokens take
// 14.2 us for 12.2.)
__device__ inline void angle_cos_sin(int pos, float inv_freq, float& c, float& s) {
  const double two_over_pi = 0.6366197723675814;
  const float two_over_pi_rest = -3.935735335e-17f;
  const double turns = inv_freq * two_over_pi;
  const float turns_rest = (float)fma((double)inv_freq, two_over_pi, -turns) + inv_freq * two_over_pi_rest;
  const double q = rint(pos * turns);
  const float x = ((float)fma((double)pos, turns, -q) + (float)pos * turns_rest) * 1.57079632679489661923f;
  const int quadrant = (int)(q - 4.0 * rint(q * 0.25)) & 3;  // q modulo 4 also where q passes 32 bits
  const float x2 = x * x;
  const float sn = x * (1.f + x2 * (-1.f / 6 + x2 * (1.f / 120 + x2 * (-1.f / 5040 + x2 * (1.f / 362880)))));
  const float cs = 1.f + x2 * (-0.5f + x2 * (1.f / 24 + x2 * (-1.f / 720 + x2 * (1.f / 40320 + x2 * (-1.f / 3628800)))));
  const float a = quadrant & 1 ? cs : sn, b = quadrant & 1 ? sn : cs;
  s = quadrant & 2 ? -a : a;
  c = (quadrant == 1 || quadrant == 2) ? -b : b;
}

template <typename T, int W>
struct Vec {
  typedef T type __attribute__((ext_vector_type(W)));
  typedef type unaligned __attribute__((aligned(sizeof(T))));
};
template <typename T>
struct Vec<T, 1> {
  typedef T type;
  typedef T unaligned;
};

enum UnitKind { TURN, TURN_ONE, PASS, PASS_ONE };

// The units of a head: R rotated channels of D, W elements to a vector.
template <int W, bool HALVES>
struct Units {
  int turn, turn_one, pass, pass_one;
  __host__ __device__ Units(int D, int R) {
    const int pairs_per_unit = HALVES ? W : W / 2;
    turn = R / 2 / pairs_per_unit;
    turn_one = R / 2 % pairs_per_unit;
    pass = (D - R) / W;
    pass_one = (D - R) % W;
  }
  __host__ __device__ int count() const { return turn + turn_one + pass + pass_one; }
};

struct RopeKernelArgs {
  RopeArgs a;
  uint32_t axis_bits[PA_ROPE_MAX_PAIRS / 16];  // pair_axis, two bits a pair: in scalar registers, unlike an array indexed by lane
  int tokens;  // per workgroup
  int groups;  // of heads that a token is split over: thread (token, group g, unit) does heads g, g + groups, ...
};

template <bool PAST_CACHES, typename V, typename VU>
__device__ inline void store(VU* p, V x) {
  if (PAST_CACHES) __builtin_nontemporal_store(x, p); else *p = x;
}

template <typename T, bool HALVES, bool APPEND, int HPT>
__global__ __launch_bounds__(THREADS) void rope_kernel(const RopeKernelArgs ka) {
  constexpr int W = 16 / sizeof(T);
  constexpr bool PAST = HPT > 4;  // stores past the caches: results that these cannot hold anyway (44 MB of fp32, kept in them: 13.9 -> 12.3 us)
  using V = typename Vec<T, W>::type;
  using VU = typename Vec<T, W>::unaligned;
  const RopeArgs& a = ka.a;
  const int D = a.rope.head_dim, R = a.rope.rotary_dim, half = R / 2;
  const Units<W, HALVES> units(D, R);
  const int U = units.count(), per_token = U * ka.groups;
  const int heads = a.Hq + a.Hk + (APPEND ? a.Hv : 0);
  const int64_t t0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ka.tokens;
  const int ntok = (int)(a.T - t0 < ka.tokens ? a.T - t0 : ka.tokens);
  if (ntok <= 0) return;

  // append: the cache row (page, slot) of each of the workgroup's tokens, -1: not stored, -2: padding behind the last sequence; worked out
  // while the first round's loads are under way
  __shared__ int64_t place[APPEND ? THREADS : 1];
  auto find_places = [&]() {
    if ((int)threadIdx.x < ntok) place[threadIdx.x] = -2;
    __syncthreads();
    for (int b = threadIdx.x; b < a.B; b += THREADS) {
      const int64_t lo = a.cu_new[b], hi = a.cu_new[b + 1];
      const int64_t first = lo > t0 ? lo : t0, last = hi < t0 + ntok ? hi : t0 + ntok;
      if (first >= last) continue;
      const int64_t len = a.seq_lens[b];
      for (int64_t t = first; t < last; ++t) {
        const int64_t pos = len - hi + t;  // hi - t tokens before the end
        int64_t at = -1;
        if (pos >= 0 && (pos >> a.page_shift) < a.table_width) {
          const int64_t page = a.page_table[(int64_t)b * a.table_width + (pos >> a.page_shift)];
          const int64_t mask = ((int64_t)1 << a.page_shift) - 1;
          if (page >= 0 && page < a.num_pages) at = ((page * a.Hk) << a.page_shift) + (pos & mask);
        }
        place[t - t0] = at;
      }
    }
    __syncthreads();
  };

  const int work = ntok * per_token;
  for (int base = 0; base < work; base += THREADS) {
    const bool live = base + (int)threadIdx.x < work;
    const int idx = live ? base + threadIdx.x : 0;
    const int tok = idx / per_token, rest = idx - tok * per_token;
    const int g = rest / U;
    int u = rest - g * U;
    const int64_t t = t0 + tok;
    UnitKind kind;
    int ca, cb;  // first channel of the unit and of its partners
    if (u < units.turn) {
      kind = TURN;
      ca = u * W;
      cb = half + ca;
    } else if ((u -= units.turn) < units.turn_one) {
      kind = TURN_ONE;
      const int i = HALVES ? units.turn * W + u : units.turn * (W / 2) + u;
      ca = HALVES ? i : 2 * i;
      cb = HALVES ? half + i : 2 * i + 1;
    } else if ((u -= units.turn_one) < units.pass) {
      kind = PASS;
      ca = cb = R + u * W;
    } else {
      kind = PASS_ONE;
      ca = cb = R + units.pass * W + (u - units.pass);
    }
    const T* src[HPT];
    V xa[HPT], xb[HPT];
#pragma unroll
    for (int i = 0; i < HPT; ++i) {
      const int h = g + i * ka.groups;
      src[i] = nullptr;
      if (!live) continue;
      if (h < a.Hq) src[i] = static_cast<const T*>(a.q) + t * a.q_stride + h * D;
      else if (h < a.Hq + a.Hk) src[i] = static_cast<const T*>(a.k) + t * a.k_stride + (h - a.Hq) * D;
      else if (APPEND && h < heads) src[i] = static_cast<const T*>(a.v) + t * a.v_stride + (h - a.Hq - a.Hk) * D;
      if (!src[i]) continue;
      if (kind == TURN || kind == PASS) {
        xa[i] = *reinterpret_cast<const VU*>(src[i] + ca);
        if (HALVES && kind == TURN) xb[i] = *reinterpret_cast<const VU*>(src[i] + cb);
      } else {
        xa[i][0] = src[i][ca];
        if (kind == TURN_ONE) xb[i][0] = src[i][cb];
      }
    }
    constexpr int N = HALVES ? W : W / 2;  // pairs of a full unit
    float cs[N], sn[N];
    if (live && (kind == TURN || kind == TURN_ONE)) {
      const int n = kind == TURN ? N : 1;
      const int pair0 = HALVES ? ca : ca / 2;  // a full unit's pairs are within one word
      uint32_t bits = ka.axis_bits[0];
      for (int w = 1; w * 32 < R; ++w) bits = pair0 >> 4 == w ? ka.axis_bits[w] : bits;
      bits >>= 2 * (pair0 & 15);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        cs[e] = 1.f;
        sn[e] = 0.f;
        if (e < n) {
          angle_cos_sin(a.positions[(int64_t)(bits >> 2 * e & 3) * a.T + t], a.inv_freq[pair0 + e], cs[e], sn[e]);
          sn[e] *= a.sign;
        }
      }
    }
    if (APPEND && base == 0) find_places();
    const int64_t at = APPEND ? place[tok] : 0;
#pragma unroll
    for (int i = 0; i < HPT; ++i) {
      const int h = g + i * ka.groups;
      if (!src[i] || (APPEND && at == -2)) continue;
      T* y;
      const bool turn = h < a.Hq + a.Hk;
      if (h < a.Hq) {
        y = static_cast<T*>(a.q_out) + t * a.q_out_stride + h * D;
      } else if (!APPEND) {
        y = static_cast<T*>(a.k_out) + t * a.k_out_stride + (h - a.Hq) * D;
      } else {
        if (at < 0) continue;
        const int hk = turn ? h - a.Hq : h - a.Hq - a.Hk;
        y = static_cast<T*>(turn ? a.k_cache : a.v_cache) + (at + ((int64_t)hk << a.page_shift)) * D;
      }
      if (kind == PASS || (kind == TURN && !turn)) {
        store<PAST>(reinterpret_cast<VU*>(y + ca), xa[i]);
        if (HALVES && kind == TURN) store<PAST>(reinterpret_cast<VU*>(y + cb), xb[i]);
      } else if (kind == PASS_ONE || !turn) {
        y[ca] = xa[i][0];
        if (kind == TURN_ONE) y[cb] = xb[i][0];
      } else if (kind == TURN) {
        V ya, yb;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float x0 = HALVES ? (float)xa[i][e] : (float)xa[i][2 * e % W];
          const float x1 = HALVES ? (float)xb[i][e] : (float)xa[i][(2 * e + 1) % W];
          const float y0 = x0 * cs[e] - x1 * sn[e], y1 = x1 * cs[e] + x0 * sn[e];  // rounded to T once
          if (HALVES) {
            ya[e] = (T)y0;
            yb[e] = (T)y1;
          } else {
            ya[2 * e % W] = (T)y0;
            ya[(2 * e + 1) % W] = (T)y1;
          }
        }
        store<PAST>(reinterpret_cast<VU*>(y + ca), ya);
        if (HALVES) store<PAST>(reinterpret_cast<VU*>(y + cb), yb);
      } else {
        const float x0 = (float)xa[i][0], x1 = (float)xb[i][0];
        y[ca] = (T)(x0 * cs[0] - x1 * sn[0]);
        y[cb] = (T)(x1 * cs[0] + x0 * sn[0]);
      }
    }
  }
}

template <typename T, bool HALVES, bool APPEND>
int launch(const RopeArgs& a, void* stream) {
  const Units<16 / (int)sizeof(T), HALVES> units(a.rope.head_dim, a.rope.rotary_dim);
  const int heads = a.Hq + a.Hk + a.Hv;
  RopeKernelArgs k{};
  k.a = a;
  for (int i = 0; i < a.rope.rotary_dim / 2; ++i) k.axis_bits[i / 16] |= (uint32_t)a.rope.pair_axis[i] << (2 * (i % 16));
  // As many heads as leave a few wavefronts to every SIMD: 8 from 2^21 units on (2^18 threads), 4 from 2^18 on.  With 2, 4 and 8 heads, whole heads turned,
  // bf16, 28 + 4 of 128: 2^17 units 5.2, 5.8, 7.3 us, 2^18 6.6, 6.5, 7.7, 2^19 10.5, 9.1, 7.7, 2^20 20, 15.9, 12.8, 2^21 37, 31, 28; fp32, 14 + 2 of 64:
  // 2^18 4.0, 4.3, 5.2, 2^19 5.3, 5.3, 5.7, 2^20 7.8, 7.5, 6.4, 2^21 14.7, 13.0, 11.3.  Below 2^21 it depends: 46 of 64 channels turned in fp32
  // (2^20.6 units) take 12.7 us with 4 and 14.0 with 8.
  const int64_t work = a.T * heads * units.count();
  const int hpt = work >= (1 << 21) ? 8 : work >= (1 << 18) ? 4 : 2;
  k.groups = (heads + hpt - 1) / hpt;
  const int per_token = units.count() * k.groups;
  k.tokens = per_token >= THREADS ? 1 : THREADS / per_token;
  const int64_t blocks = (a.T + k.tokens - 1) / k.tokens;
  const unsigned gx = (unsigned)(blocks < MAX_GRID_X ? blocks : MAX_GRID_X);
  const unsigned gy = (unsigned)((blocks + gx - 1) / gx);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (hpt == 8) rope_kernel<T, HALVES, APPEND, 8><<<dim3(gx, gy), THREADS, 0, st>>>(k);
  else if (hpt == 4) rope_kernel<T, HALVES, APPEND, 4><<<dim3(gx, gy), THREADS, 0, st>>>(k);
  else rope_kernel<T, HALVES, APPEND, 2><<<dim3(gx, gy), THREADS, 0, st>>>(k);
  return (int)hipGetLastError();
}

template <bool APPEND>
int dispatch(const RopeArgs& a, void* stream) {
  const bool halves = a.rope.layout == PA_ROPE_HALVES;
  if (a.dtype == PA_BF16) return halves ? launch<__bf16, true, APPEND>(a, stream) : launch<__bf16, false, APPEND>(a, stream);
  return halves ? launch<float, true, APPEND>(a, stream) : launch<float, false, APPEND>(a, stream);
}

}  // namespace

int launch_rope(const RopeArgs& a, void* stream) { return dispatch<false>(a, stream); }
int launch_append(const RopeArgs& a, void* stream) { return dispatch<true>(a, stream); }

}  // namespace pa
