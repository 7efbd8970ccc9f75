// Scores of logits rows: log probability and rank of a given token, entropy, top alternatives, in one pass.
//
//   m = max x,  S = sum e^(x - m),  T = sum (x - m) e^(x - m)
//   log p_t = (x_t - m) - log S,    H = log S - T / S
// A thread keeps (m, S, T) of its share and rescales when its maximum moves: with m' > m,
//   S' = f S, T' = f (T + (m - m') S), f = e^(m - m').  T uses x - m, not x: the entropy of a sure row, near 0, would
// otherwise be the difference of two large numbers.  Exponentials in base 2 (one multiply in front of ex2.approx, relative
// error 2^-22); sums in fp32 over short per-thread shares.
// Alternatives: a warp keeps the best 32 of what it has seen as sorted 64-bit keys (value in sortable form, then the
// complement of the id: equal values lowest id first), one a lane.  A value is only looked at when it exceeds the top-th
// key; of random logits few do (top * ln(n / top) per warp).  Many at once (the first values of a row, ascending logits)
// are sorted across the warp and merged, few are inserted one by one.
#pragma once
#include <cuda_fp16.h>

#include "fm_common.cuh"
#include "fm_ptx.cuh"
#include "../../include/flashmesh.h"

namespace lp {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f, LOWEST = -3.402823466e38f;

struct Args {
  const void* x;
  const int* tokens;
  float *logprob, *entropy;
  int* rank;
  int* top_ids;
  float* top_logprobs;
  int64_t stride;                       // elements
  int rows, vocab, top;
};

__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T> __device__ inline float load1(const T* p);
template <> __device__ inline float load1<float>(const float* p) { return *p; }
template <> __device__ inline float load1<bf16>(const bf16* p) { return __bfloat162float(*p); }
template <> __device__ inline float load1<__half>(const __half* p) { return __half2float(*p); }
template <typename T> struct Vec { static constexpr int N = 16 / sizeof(T); };
__device__ inline void unpack(const uint4& v, float (&x)[4], const float*) {
  x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
__device__ inline void unpack(const uint4& v, float (&x)[8], const bf16*) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ inline void unpack(const uint4& v, float (&x)[8], const __half*) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i])); x[2 * i] = f.x; x[2 * i + 1] = f.y; }
}

// Key of a value: larger keys rank first; 0 = nothing.  (-0 and +0 are one value; a NaN ranks below everything.)
__device__ inline uint64_t key_of(float x, int id) {
  if (x != x) return (uint64_t)(uint32_t)~id;
  const int b = __float_as_int(x + 0.f);
  const uint32_t u = (uint32_t)(b ^ ((b >> 31) & 0x7fffffff)) ^ 0x80000000u;
  return ((uint64_t)u << 32) | (uint32_t)~id;
}
__device__ inline int key_id(uint64_t k) { return (int)~(uint32_t)k; }
__device__ inline float key_value(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  if (u < 0x007fffffu) return __int_as_float(0x7fc00000);    // below the key of -inf: a NaN
  const int s = (int)(u ^ 0x80000000u);
  return __int_as_float(s ^ ((s >> 31) & 0x7fffffff));
}

__device__ inline uint64_t kmax(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ inline uint64_t kmin(uint64_t a, uint64_t b) { return a < b ? a : b; }
// descending order across the lanes of a bitonic sequence
__device__ inline uint64_t bitonic_tail(uint64_t k, int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const uint64_t q = __shfl_xor_sync(0xffffffffu, k, o);
    k = (lane & o) ? kmin(k, q) : kmax(k, q);
  }
  return k;
}
__device__ inline uint64_t warp_sort(uint64_t k, int lane) {
#pragma unroll
  for (int n = 2; n <= 32; n <<= 1)
#pragma unroll
    for (int o = n >> 1; o > 0; o >>= 1) {
      const uint64_t q = __shfl_xor_sync(0xffffffffu, k, o);
      const bool keep_max = ((lane & o) == 0) == ((lane & n) == 0 || n == 32);
      k = keep_max ? kmax(k, q) : kmin(k, q);
    }
  return k;
}
// the best 32 of two lists in descending order
__device__ inline uint64_t merge_lists(uint64_t a, uint64_t b, int lane) {
  return bitonic_tail(kmax(a, __shfl_sync(0xffffffffu, b, 31 - lane)), lane);
}
// take in one candidate a lane (0 = none)
__device__ inline void push(uint64_t& list, uint64_t& bar, uint64_t cand, int top, int lane) {
  unsigned m = __ballot_sync(0xffffffffu, cand > bar);
  if (m == 0) return;
  if (__popc(m) > 5) {
    list = merge_lists(list, warp_sort(cand > bar ? cand : 0ull, lane), lane);
  } else {
    while (m != 0) {
      const uint64_t k = __shfl_sync(0xffffffffu, cand, __ffs(m) - 1);
      m &= m - 1;
      const int at = __popc(__ballot_sync(0xffffffffu, list > k));
      const uint64_t up = __shfl_up_sync(0xffffffffu, list, 1);
      list = lane < at ? list : (lane == at ? k : up);
    }
  }
  bar = __shfl_sync(0xffffffffu, list, top - 1);
}

struct Sums { float m, s, t; };
__device__ inline void rescale(Sums& a, float m) {           // m >= a.m
  if (a.s != 0.f) {
    const float d = a.m - m, f = ex2(d * LOG2E);
    a.t = (a.t + d * a.s) * f;
    a.s *= f;
    if (f == 0.f) a.t = 0.f;                                 // (0 * inf where d overflows)
  }
  a.m = m;
}
__device__ inline void merge(Sums& a, Sums b) {
  const float m = fmaxf(a.m, b.m);
  rescale(a, m);
  rescale(b, m);
  a.s += b.s;
  a.t += b.t;
}
__device__ inline void add(Sums& a, float x) {               // x <= a.m, or a NaN
  const float d = x - a.m, e = ex2(d * LOG2E);
  a.s += e;
  a.t += e == 0.f ? 0.f : d * e;
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS) rows_kernel(const Args a) {
  constexpr int NW = THREADS / 32, N = Vec<T>::N;
  __shared__ Sums s_sum[NW];
  __shared__ int s_rank[NW];
  __shared__ uint64_t s_list[NW][32];
  const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.stride;
  const int token = a.tokens != nullptr ? a.tokens[row] : -1;
  const bool given = token >= 0 && token < a.vocab;
  const float xt = given ? load1(x + token) : __int_as_float(0x7fc00000);      // (nothing exceeds a NaN)
  Sums sum{LOWEST, 0.f, 0.f};
  int above = 0;
  uint64_t list = 0, bar = 0;
  auto one = [&](float v, int id, bool there) {              // a warp in step; v counts where `there`
    if (there) {
      if (v > sum.m) rescale(sum, v);
      add(sum, v);
      above += v > xt;
    }
    if (a.top > 0) push(list, bar, there ? key_of(v, id) : 0ull, a.top, lane);
  };
  // elements in front of the first 16-byte boundary, whole vectors, the rest
  const int head = min(a.vocab, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
  const int n_vec = (a.vocab - head) / N, tail0 = head + n_vec * N;
  if (warp == 0) one(lane < head ? load1(x + lane) : 0.f, lane, lane < head);
  if (warp == NW - 1) one(lane < a.vocab - tail0 ? load1(x + tail0 + lane) : 0.f, tail0 + lane, lane < a.vocab - tail0);
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  constexpr int U = 4;                                       // vectors in flight a thread
  for (int i0 = warp * 32; i0 < n_vec; i0 += U * THREADS) {
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * THREADS + lane;
      if (i < n_vec) raw[u] = __ldg(xv + i);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * THREADS + lane;
      if (i0 + u * THREADS >= n_vec) break;                  // the same for the warp
      const bool there = i < n_vec;
      float v[N];
      float mx = -INFINITY;
      if (there) {
        unpack(raw[u], v, static_cast<const T*>(nullptr));
#pragma unroll
        for (int j = 0; j < N; ++j) mx = fmaxf(mx, v[j]);
        if (mx > sum.m) rescale(sum, mx);
#pragma unroll
        for (int j = 0; j < N; ++j) { add(sum, v[j]); above += v[j] > xt; }
      }
      // (the bar is the smallest key that still counts: a value can only enter where its key, not below the value alone, does)
      if (a.top > 0 && __any_sync(0xffffffffu, there && (key_of(mx, 0) > bar || bar < (1ull << 32)))) {
#pragma unroll
        for (int j = 0; j < N; ++j) push(list, bar, there ? key_of(v[j], head + i * N + j) : 0ull, a.top, lane);
      }
    }
  }
  // ---- the warp's sums, then the block's
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b;
    b.m = __shfl_xor_sync(0xffffffffu, sum.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, sum.s, o);
    b.t = __shfl_xor_sync(0xffffffffu, sum.t, o);
    // the same order of operands in both lanes: the same bits
    if (lane & o) { merge(b, sum); sum = b; } else merge(sum, b);
  }
  above = __reduce_add_sync(0xffffffffu, above);
  if (lane == 0) { s_sum[warp] = sum; s_rank[warp] = above; }
  s_list[warp][lane] = list;
  __syncthreads();
  if (warp != 0) return;
  for (int w = 1; w < NW; ++w) {
    merge(sum, s_sum[w]);
    above += s_rank[w];
    if (a.top > 0) list = merge_lists(list, s_list[w][lane], lane);
  }
  const bool nothing = sum.s == 0.f;                         // a row of -inf alone
  const float log_s = logf(sum.s);
  if (lane == 0) {
    if (a.logprob != nullptr) a.logprob[row] = !given || nothing ? -INFINITY : (xt - sum.m) - log_s;
    if (a.entropy != nullptr) a.entropy[row] = nothing ? 0.f : log_s - sum.t / sum.s;
    if (a.rank != nullptr) a.rank[row] = given ? above : -1;
  }
  if (lane < a.top) {
    if (a.top_ids != nullptr) a.top_ids[(int64_t)row * a.top + lane] = key_id(list);
    if (a.top_logprobs != nullptr) a.top_logprobs[(int64_t)row * a.top + lane] = nothing ? -INFINITY : (key_value(list) - sum.m) - log_s;
  }
}

}  // namespace lp
