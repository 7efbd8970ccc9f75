// Scores of logits rows: log probability and rank of a given token, entropy, top alternatives, in one pass.
//
//   m = max x,  S = sum e^(x - m),  T = sum (x - m) e^(x - m)
//   log p_t = (x_t - m) - log S,    H = log S - T / S
// with the exponentials in base 2, d = (x - m) log2 e (the difference first: values up to the type's largest and lowest stay
// finite).  A thread keeps (m, S, T) of its share and rescales when its maximum moves: S' = f S, T' = f (T + d S), f = 2^d,
// d = (m - m') log2 e.  T uses differences, not values: the entropy of a sure row, near 0, would otherwise be the
// difference of two large numbers.  ex2.approx has a relative error of 2^-22; sums in fp32 over short per-thread shares, in pairs (fma.f32x2).
// Alternatives: keys of 64 bits, the value in sortable form, then the complement of the id (equal values lowest id first).
// Of any `top` lanes, or threads, the least of their maxima is a bound that `top` values of the row reach: the top-th largest of
// the maxima of a row's first values is found by sorting, and only values that reach it are collected; in random order
// that is top * (values of the row / values looked at) of them.  The collected ones are sorted 32 at a time across warps.
// Where they do not fit (rising logits, many equal ones) the row is read again: a warp keeps the best 32 of its share
// as a sorted list, one a lane, and takes in what exceeds its top-th.
//
// Rows are read by plain loads: a kernel here is resident before the launch that writes its logits has ended, so they are not
// read-only for as long as it runs (a non-coherent load may be moved across the wait for that launch).
//
// Short rows (up to 2048 values) live in the registers of a warp; long ones take a block, the threads copying
// 2048 or 4096 vectors ahead, each into shared memory of its own (cp.async: no barrier, nothing waits for a neighbour).
// Bound: of 16-bit values the special-function units, an exponential each, then the latency of a row's start and end: 512 rows of
// 128011 take 39 us, with 20 alternatives 45 (20 at the copy rate; an SM has up to four rows, 16 us of exponentials); of
// fp32 57 us (70 % of the copy rate).  40000 rows of 1027 fp32: 33 us (76 %), with 20 alternatives 72: the sorting of each
// row's list.  Ten rows of 1027: 8 us, a launch and two round trips to memory.
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

// two fp32 in one register pair
__device__ inline uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ inline float2 halves(uint64_t r) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ inline uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ inline uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ inline uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ inline float max_nan(float a, float b) {          // a NaN stays one
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ inline float exceeds(float a, float b) {          // 1 or 0
  float r;
  asm("set.gt.f32.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct Sums { float m, s, t; };         // maximum, S, T (of d)
__device__ inline void rescale(Sums& a, float m) {           // m >= a.m
  if (a.s != 0.f) {
    const float d = (a.m - m) * LOG2E, f = ex2(d);
    a.t = f == 0.f ? 0.f : (a.t + d * a.s) * f;
    a.s *= f;
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
// A difference below this adds nothing (2^-150 is flushed to zero); the bound keeps -inf out of the product d * 2^d.
constexpr float DEEP = -150.f;


// ---- a row's results from its sums, the count above the token, and the list (one key a lane)
__device__ inline void write_row(const Args& a, int row, int lane, const Sums& sum, bool given, float xt, int above, uint64_t list) {
  const bool nothing = sum.s == 0.f;                         // a row of -inf alone
  const float log_s = log2f(sum.s);
  auto logp = [&](float v) { return nothing ? -INFINITY : (v - sum.m) - log_s * LN2; };
  if (lane == 0) {
    if (a.logprob != nullptr) a.logprob[row] = given ? logp(xt) : -INFINITY;
    if (a.entropy != nullptr) a.entropy[row] = nothing ? 0.f : (log_s - sum.t / sum.s) * LN2;
    if (a.rank != nullptr) a.rank[row] = given ? above : -1;
  }
  if (lane < a.top) {
    if (a.top_ids != nullptr) a.top_ids[(int64_t)row * a.top + lane] = key_id(list);
    if (a.top_logprobs != nullptr) a.top_logprobs[(int64_t)row * a.top + lane] = logp(key_value(list));
  }
}
// elements in front of the first 16-byte boundary, whole vectors behind them, where the rest starts
template <typename T>
struct Cut {
  int head, n_vec, tail0;
  __device__ Cut(const T* x, int vocab) {
    head = min(vocab, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
    n_vec = (vocab - head) / Vec<T>::N;
    tail0 = head + n_vec * Vec<T>::N;
  }
  // the elements outside the vectors, one a lane (fewer than 16): id, or -1
  __device__ int loose(int lane, int vocab) const {
    const int i = lane < head ? lane : tail0 + (lane - head);
    return lane < head + (vocab - tail0) ? i : -1;
  }
};
// sortable form of a value for bounds: monotonic, 0 for a NaN
__device__ inline uint32_t order_of(float x) { return (uint32_t)(key_of(x, 0) >> 32); }
__device__ inline uint32_t sort32(uint32_t k, int lane) {    // descending across the lanes
#pragma unroll
  for (int n = 2; n <= 32; n <<= 1)
#pragma unroll
    for (int o = n >> 1; o > 0; o >>= 1) {
      const uint32_t q = __shfl_xor_sync(0xffffffffu, k, o);
      const bool keep_max = ((lane & o) == 0) == ((lane & n) == 0 || n == 32);
      k = keep_max ? max(k, q) : min(k, q);
    }
  return k;
}
__device__ inline uint32_t merge32(uint32_t a, uint32_t b, int lane) {
  uint32_t k = max(a, __shfl_sync(0xffffffffu, b, 31 - lane));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const uint32_t q = __shfl_xor_sync(0xffffffffu, k, o);
    k = (lane & o) ? min(k, q) : max(k, q);
  }
  return k;
}
// the k-th largest across the lanes, k >= 1
__device__ inline uint32_t kth32(uint32_t k32, int k, int lane) {
  if (k > 6) return __shfl_sync(0xffffffffu, sort32(k32, lane), k - 1);
  uint32_t m = 0;
  for (int i = 0; i < k; ++i) {                              // (a sort takes about as long as seven of these)
    m = __reduce_max_sync(0xffffffffu, k32);
    if (lane == __ffs(__ballot_sync(0xffffffffu, k32 == m)) - 1) k32 = 0;
  }
  return m;
}
// `total` distinct keys in shared memory, in descending order across the lanes: the best 32 of them
__device__ inline uint64_t sort_keys(uint64_t* keys, int total, int lane) {
  if (total <= 12) {                                         // by counting the larger ones
    const uint64_t mine = lane < total ? keys[lane] : 0ull;
    int r = 0;
    for (int j = 0; j < total; ++j) r += keys[j] > mine;
    __syncwarp();
    if (lane < total) keys[r] = mine;
    __syncwarp();
    return lane < total ? keys[lane] : 0ull;
  }
  uint64_t list = warp_sort(lane < total ? keys[lane] : 0ull, lane);
  for (int i = 32; i < total; i += 32) list = merge_lists(list, warp_sort(i + lane < total ? keys[i + lane] : 0ull, lane), lane);
  return list;
}
// A pair of values into the sums (differences to sum.m, which is not below them).
__device__ inline void add_pair(uint64_t& s2, uint64_t& t2, float x0, float x1, uint64_t nm) {
  const float2 d = halves(mul2(add2(pair(x0, x1), nm), pair(LOG2E, LOG2E)));
  const float d0 = max_nan(d.x, DEEP), d1 = max_nan(d.y, DEEP);
  const uint64_t e = pair(ex2(d0), ex2(d1));
  s2 = add2(s2, e);
  t2 = fma2(pair(d0, d1), e, t2);
}
__device__ inline Sums warp_sums(Sums sum, int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b;
    b.m = __shfl_xor_sync(0xffffffffu, sum.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, sum.s, o);
    b.t = __shfl_xor_sync(0xffffffffu, sum.t, o);
    // the same order of operands in both lanes: the same bits
    if (lane & o) { merge(b, sum); sum = b; } else merge(sum, b);
  }
  return sum;
}

// The best 32 of elements first, first + step, ... (a warp takes 32 neighbours at a time): exact for any order of values
template <typename T>
__device__ __noinline__ uint64_t list_of(const T* x, int vocab, int first, int step, int top, int lane) {
  uint64_t list = 0, bar = 0;
  for (unsigned i0 = first; i0 < (unsigned)vocab; i0 += step) {    // (unsigned: a step behind the last of 2^31 - 1 values)
    const unsigned i = i0 + lane;
    push(list, bar, i < (unsigned)vocab ? key_of(load1(x + i), (int)i) : 0ull, top, lane);
  }
  return list;
}

// ---- short rows: a warp each, the row in registers (R vectors a lane)
constexpr int SHORT_WARPS = 4, SHORT_CAP = 256;
template <typename T, int R>
__global__ void __launch_bounds__(32 * SHORT_WARPS) short_kernel(const Args a) {
  constexpr int N = Vec<T>::N;
  __shared__ uint64_t s_cand[SHORT_WARPS][SHORT_CAP];
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * SHORT_WARPS + warp;
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.stride;
  const Cut<T> cut(x, a.vocab);
  const uint4* xv = reinterpret_cast<const uint4*>(x + cut.head);
  uint4 raw[R];
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r * 32 + lane < cut.n_vec) raw[r] = xv[r * 32 + lane];
  const int loose = cut.loose(lane, a.vocab);
  const float xl = loose >= 0 ? load1(x + loose) : -INFINITY;
  const int token = a.tokens != nullptr ? a.tokens[row] : -1;
  const bool given = token >= 0 && token < a.vocab;
  const float xt = given ? load1(x + token) : __int_as_float(0x7fc00000);      // (nothing exceeds a NaN)
  float mx = xl != xl ? -INFINITY : xl;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r * 32 + lane < cut.n_vec) {
      float v[N];
      unpack(raw[r], v, static_cast<const T*>(nullptr));
#pragma unroll
      for (int j = 0; j < N; j += 2) mx = max3(mx, v[j], v[j + 1]);
    }
  Sums sum{fmaxf(warp_max(mx), LOWEST), 0.f, 0.f};
  const uint64_t nm = pair(-sum.m, -sum.m);
  uint64_t s2 = 0, t2 = 0;
  uint64_t n2 = pair(exceeds(xl, xt), 0.f);
  if (loose >= 0) add_pair(s2, t2, xl, -INFINITY, nm);
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r * 32 + lane < cut.n_vec) {
      float v[N];
      unpack(raw[r], v, static_cast<const T*>(nullptr));
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        add_pair(s2, t2, v[j], v[j + 1], nm);
        n2 = add2(n2, pair(exceeds(v[j], xt), exceeds(v[j + 1], xt)));
      }
    }
  const float2 s = halves(s2), t = halves(t2);
  sum.s = warp_sum(s.x + s.y);                               // (one maximum for all lanes: the parts only add)
  sum.t = warp_sum(t.x + t.y);
  const int above = __reduce_add_sync(0xffffffffu, (int)(halves(n2).x + halves(n2).y));
  uint64_t list = 0;
  if (a.top > 0) {
    const uint32_t bound = kth32(order_of(mx), a.top, lane);
    // what reaches the bound; a bound at or below -inf says nothing.  (Counted, then written behind the lanes in front: a
    // counter in shared memory instead kept the row's registers alive in the branch, 86 against 72 us for 40000 rows of 1027.)
    const bool some = bound > order_of(-INFINITY);
    const float least = some ? key_value((uint64_t)bound << 32) : INFINITY;
    int mine = loose >= 0 && xl >= least;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r * 32 + lane < cut.n_vec) {
        float v[N];
        unpack(raw[r], v, static_cast<const T*>(nullptr));
#pragma unroll
        for (int j = 0; j < N; ++j) mine += v[j] >= least;
      }
    int at = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, at, o);
      if (lane >= o) at += y;
    }
    const int total = __shfl_sync(0xffffffffu, at, 31);
    at -= mine;
    if (!some || total > SHORT_CAP) {
      list = list_of(x, a.vocab, 0, 32, a.top, lane);
    } else {
      uint64_t* cand = s_cand[warp];
      if (mine > 0) {
        if (loose >= 0 && xl >= least) cand[at++] = key_of(xl, loose);
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (r * 32 + lane < cut.n_vec) {
            float v[N];
            unpack(raw[r], v, static_cast<const T*>(nullptr));
#pragma unroll
            for (int j = 0; j < N; ++j)
              if (v[j] >= least) cand[at++] = key_of(v[j], cut.head + (r * 32 + lane) * N + j);
          }
      }
      __syncwarp();
      list = sort_keys(cand, total, lane);
    }
  }
  write_row(a, row, lane, sum, given, xt, above, list);
}

// ---- long rows: a block each
constexpr int LONG_CAP = 1024;
template <typename T, int THREADS, int AHEAD>
__global__ void __launch_bounds__(THREADS) long_kernel(const Args a) {
  constexpr int NW = THREADS / 32, N = Vec<T>::N, GR = AHEAD / 2;
  extern __shared__ uint4 s_ring[];                          // [AHEAD][THREADS]
  __shared__ int s_vec[LONG_CAP];                            // vectors with a value that reaches the bound
  __shared__ uint64_t s_cand[LONG_CAP];                      // keys of such values
  __shared__ uint64_t s_list[NW][32];
  __shared__ uint32_t s_bound[NW][32];
  __shared__ Sums s_sum[NW];
  __shared__ int s_rank[NW];
  __shared__ int s_count, s_keys;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* x = static_cast<const T*>(a.x) + (int64_t)row * a.stride;
  const Cut<T> cut(x, a.vocab);
  const uint4* xv = reinterpret_cast<const uint4*>(x + cut.head);
  const int n = (cut.n_vec - tid + THREADS - 1) / THREADS;   // this thread's vectors (0 or less: none)
  // requested in groups of GR, two of them in flight
  const uint32_t ring = ptx::smem_u32(s_ring + tid);
  const uint4* next = xv + tid;
  auto request = [&](int k, uint32_t at) {                   // vectors k .. k + GR - 1 of the thread into places from `at`
#pragma unroll
    for (int j = 0; j < GR; ++j)
      if (k + j < n) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + j * THREADS * 16), "l"(next + j * THREADS) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
    next += GR * THREADS;
  };
  request(0, ring);
  request(GR, ring + GR * THREADS * 16);
  const int token = a.tokens != nullptr ? a.tokens[row] : -1;
  const bool given = token >= 0 && token < a.vocab;
  const float xt = given ? load1(x + token) : __int_as_float(0x7fc00000);      // (nothing exceeds a NaN)
  const int loose = warp == 0 ? cut.loose(lane, a.vocab) : -1;
  const float xl = loose >= 0 ? load1(x + loose) : -INFINITY;
  if (tid == 0) s_count = s_keys = 0;
  // the maxima of what has been requested: their largest is the reference of the sums, their top-th the bound
  asm volatile("cp.async.wait_all;" ::: "memory");
  float mx = xl != xl ? -INFINITY : xl;
#pragma unroll
  for (int k = 0; k < AHEAD; ++k)
    if (k < n) {
      float v[N];
      unpack(s_ring[k * THREADS + tid], v, static_cast<const T*>(nullptr));
#pragma unroll
      for (int j = 0; j < N; j += 2) mx = max3(mx, v[j], v[j + 1]);
    }
  uint32_t bound = order_of(mx);
  if (a.top > 1) {
    bound = sort32(bound, lane);
  } else {
    const uint32_t most = __reduce_max_sync(0xffffffffu, bound);             // (by all lanes at one place, then chosen)
    bound = lane == 0 ? most : 0u;
  }
  s_bound[warp][lane] = bound;
  for (int o = NW / 2; o > 0; o >>= 1) {
    __syncthreads();
    if (warp < o) {
      bound = merge32(bound, s_bound[warp + o][lane], lane);
      s_bound[warp][lane] = bound;
    }
  }
  __syncthreads();
  Sums sum{fmaxf(key_value((uint64_t)s_bound[0][0] << 32), LOWEST), 0.f, 0.f};
  bound = a.top > 0 ? s_bound[0][a.top - 1] : 0u;
  const bool some = bound > order_of(-INFINITY);             // (a bound at or below -inf says nothing)
  const float least = some ? key_value((uint64_t)bound << 32) : INFINITY;      // what reaches it is collected
  // (the order of the collected does not matter: they are sorted)
  auto collect = [&](float v, int id) {
    const int at = atomicAdd(&s_keys, 1);
    if (at < LONG_CAP) s_cand[at] = key_of(v, id);
  };
  uint64_t s2 = 0, t2 = 0, n2 = 0, nm = pair(-sum.m, -sum.m);
  auto vector = [&](const uint4& raw, int k) {
    float v[N];
    unpack(raw, v, static_cast<const T*>(nullptr));
    float mx = fmaxf(v[0], v[1]);
#pragma unroll
    for (int j = 2; j < N; j += 2) mx = max3(mx, v[j], v[j + 1]);
    if (mx > sum.m) {                                        // seldom: above the largest of the first values
      const float2 s = halves(s2), t = halves(t2);
      sum.s = s.x + s.y;
      sum.t = t.x + t.y;
      rescale(sum, mx);
      s2 = pair(sum.s, 0.f); t2 = pair(sum.t, 0.f); nm = pair(-sum.m, -sum.m);
    }
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      add_pair(s2, t2, v[j], v[j + 1], nm);
      n2 = add2(n2, pair(exceeds(v[j], xt), exceeds(v[j + 1], xt)));
    }
    if (mx >= least) {                                       // noted, and read again below: a third of the warps' vectors has one
      const int at = atomicAdd(&s_count, 1);
      if (at < LONG_CAP) s_vec[at] = k * THREADS + tid;
    }
  };
  uint32_t at = ring;
  for (int k = 0; k < n; k += GR) {
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    uint4 raw[GR];
#pragma unroll
    for (int j = 0; j < GR; ++j)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw[j].x), "=r"(raw[j].y), "=r"(raw[j].z), "=r"(raw[j].w) : "r"(at + j * THREADS * 16) : "memory");
    if (k + GR <= n) {
#pragma unroll
      for (int j = 0; j < GR; ++j) vector(raw[j], k + j);
    } else {
      for (int j = 0; j < n - k; ++j) {                      // the last group
        uint4 r = raw[0];
#pragma unroll
        for (int q = 1; q < GR; ++q) if (q == j) r = raw[q];
        vector(r, k + j);
      }
    }
    request(k + AHEAD, at);                                  // (behind the reads of their places, by the same thread)
    at = at == ring ? ring + GR * THREADS * 16 : ring;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  sum.s = halves(s2).x + halves(s2).y;
  sum.t = halves(t2).x + halves(t2).y;
  int above = (int)(halves(n2).x + halves(n2).y);            // (exact: a thread has far fewer than 2^24 values)
  if (loose >= 0) {
    s2 = pair(sum.s, 0.f); t2 = pair(sum.t, 0.f);            // (not above the maximum: it was among the first values)
    add_pair(s2, t2, xl, -INFINITY, pair(-sum.m, -sum.m));
    sum.s = halves(s2).x + halves(s2).y;
    sum.t = halves(t2).x + halves(t2).y;
    above += xl > xt;
    if (xl >= least) collect(xl, loose);
  }
  sum = warp_sums(sum, lane);
  above = __reduce_add_sync(0xffffffffu, above);
  if (lane == 0) { s_sum[warp] = sum; s_rank[warp] = above; }
  __syncthreads();
  uint64_t list = 0;
  if (a.top > 0) {
    const int vectors = s_count;
    if (vectors <= LONG_CAP) {
      for (int i = tid; i < vectors; i += THREADS) {
        float v[N];
        unpack(xv[s_vec[i]], v, static_cast<const T*>(nullptr));
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (v[j] >= least) collect(v[j], cut.head + s_vec[i] * N + j);
      }
    }
    __syncthreads();
    const int total = s_keys;
    int lists = NW;                                          // warps that hold one
    if (!some || vectors > LONG_CAP || total > LONG_CAP) {
      list = list_of(x, a.vocab, warp * 32, THREADS, a.top, lane);
    } else {
      for (int i = warp * 32; i < total; i += THREADS) {
        const uint64_t l = sort_keys(s_cand + i, min(32, total - i), lane);
        list = i == warp * 32 ? l : merge_lists(list, l, lane);
      }
      lists = min(NW, (total + 31) >> 5);
    }
    s_list[warp][lane] = list;
    for (int o = NW / 2; o > 0; o >>= 1) {                   // the warps' lists, in pairs
      if (lists <= o) continue;                              // (the same for the block)
      __syncthreads();
      if (warp < o) {
        list = merge_lists(list, s_list[warp + o][lane], lane);
        s_list[warp][lane] = list;
      }
    }
  }
  if (warp != 0) return;
  sum = s_sum[0];
  above = s_rank[0];
  for (int w = 1; w < NW; ++w) {
    merge(sum, s_sum[w]);
    above += s_rank[w];
  }
  write_row(a, row, lane, sum, given, xt, above, list);
}

}  // namespace lp
