// Attention of trees of drafted tokens over a paged cache, and the walk that accepts a path.
//
// A tile is what shares keys: the query rows (nodes x heads of the group) of one sequence and kv-head, 16 of them.  Its keys
// come in chunks of C: conditioning slots, the window's slots (or all cached ones), the nodes.  The launch is one CTA per
// SM whatever the lengths: the chunks of all tiles, one tile after the other, are cut into equal shares (their total is
// known on the device alone), so ragged batches are balanced without the host.  A cut falls inside a tile at most once per CTA; the
// parts of a cut tile go to a scratch buffer and a second small launch merges them in order.
// Loading: four warps copy 16 bytes a thread straight into swizzled shared memory (cp.async: page, head and slot strides
// are free, what is not there is filled with zeros), a ring of stages ahead of the four warps that multiply; page ids are
// fetched a chunk ahead.  The multiplying warps each own a slice of every chunk and their own running maximum, sum
// and output (base 2), merged at the end of a tile.
// Ancestors: reach[i], a bit per node, by pointer doubling over the parents (log2 of the depth rounds).
// Values a row does not see have no effect on it: scores are replaced by -inf; values that are not finite in chunks
// where some row does not see all keys are taken out of the product and added to the rows that do see them.
#pragma once
#include <cuda_fp16.h>

#include "fm_common.cuh"
#include "fm_ptx.cuh"
#include "../../include/flashmesh.h"

namespace tr {

constexpr int CTAS = 148;               // a B200 has as many SMs; the workspace is laid out for them
constexpr int WORDS = FM_MAX_TREE_NODES / 32;

struct Div {                            // division of 0 <= n < 2^31 by a constant
  uint32_t mul; int shift, d;
  __device__ int operator()(int n) const { return d == 1 ? n : (int)(__umulhi((uint32_t)n, mul) >> shift); }
};

struct Args {
  const void *q, *k_new, *v_new;
  void* out;
  float* lse;
  int64_t q_row, new_row, out_row;      // elements
  const char *k, *v;                    // the layer's cache
  int64_t page, head, slot;             // elements
  const int *table, *lens, *seqs, *row_off, *parent;
  int* status;
  float* part;                          // [CTAS * 2][ROWS][DH + 2]
  int4* desc;                           // [CTAS]: sequence, kv-head, tile, parts of the tile that starts here and is cut
  Div page_div;
  int n_pages, max_pages, max_seqs, batch, H, Hkv, G, max_nodes, max_len, window, n_prefix;
  float scale_log2;
};

// ---- element types
__device__ inline void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bf16) { ptx::mma_bf16_16816(d, a, b0, b1); }
__device__ inline void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ inline uint32_t pack(float x, float y, bf16) { return ptx::pack_bf16(x, y); }
__device__ inline uint32_t pack(float x, float y, __half) {
  const __half2 v = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ inline float2 unpack(uint32_t v, bf16) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ inline float2 unpack(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
// halves of a word whose exponent is all ones -> 0; `bad` is set when there was one
template <typename T>
__device__ inline uint32_t finite_part(uint32_t v, bool& bad) {
  constexpr uint32_t E = sizeof(T) == 2 && __is_same(T, bf16) ? 0x7f80u : 0x7c00u;
  if ((v & E) == E) { v &= 0xffff0000u; bad = true; }
  if (((v >> 16) & E) == E) { v &= 0x0000ffffu; bad = true; }
  return v;
}

__device__ inline float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ inline void cp16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ inline void cp_arrive(uint64_t* bar) {            // when this thread's copies so far have landed
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(ptx::smem_u32(bar)) : "memory");
}

// ---- what a sequence asks for
struct Seq {
  int r0, n, len, pre, lo, seq;         // first row, nodes, cached positions; slots [0, pre) and [lo, len) are seen by some row
  int n_pre, n_main, chunks, tiles;     // chunks of the two ranges, all chunks, query tiles per kv-head
};
template <int C, int ROWS>
__device__ inline Seq sequence(const Args& a, int b) {
  Seq s;
  s.r0 = a.row_off[b];
  s.n = a.row_off[b + 1] - s.r0;
  s.n = s.r0 < 0 || s.n < 0 ? 0 : min(s.n, a.max_nodes);
  s.seq = a.seqs != nullptr ? a.seqs[b] : b;
  s.len = s.seq >= 0 && s.seq < a.max_seqs ? max(0, min(a.lens[s.seq], a.max_len)) : 0;
  s.pre = min(a.n_prefix, s.len);
  s.lo = a.window > 0 ? max(s.pre, s.len - a.window + 1) : s.pre;
  s.lo = min(s.lo, s.len);
  if (s.lo == s.pre) { s.pre = 0; s.lo = 0; }                // one range
  s.n_pre = (s.pre + C - 1) / C;
  s.n_main = (s.len - s.lo + C - 1) / C;
  s.chunks = s.n_pre + s.n_main + (s.n + C - 1) / C;
  s.tiles = (s.n * a.G + ROWS - 1) / ROWS;
  return s;
}

// ---- the cut of all chunks into shares
struct Plan {
  const long long* base;                // [batch + 1] chunks in front of a sequence's
  const int* tile_base;                 // [batch + 1] tiles in front of a sequence's
  int batch;
  long long total, share;
  bool whole;                           // CTA i takes tile i: nothing is cut
};
struct Place { int b; long long tile; int off; };            // sequence, tile of the sequence (kv-head * tiles + tile), chunk
// last sequence whose first chunk (tile) is not behind x, and that has any
template <typename V>
__device__ inline int find(const V* base, int batch, long long x) {
  int lo = 0, hi = batch;                                    // base[lo] <= x < base[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((long long)base[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}
// first chunk of CTA i's share.  A cut close to the border of a tile moves there: the tile stays whole.
template <int C, int ROWS>
__device__ inline long long boundary(const Args& a, const Plan& p, int i) {
  const long long x = p.share * i;
  if (i <= 0) return 0;
  if (x >= p.total) return p.total;
  const int b = find(p.base, p.batch, x);
  const Seq s = sequence<C, ROWS>(a, b);
  const int off = (int)((x - p.base[b]) % s.chunks);
  const long long near = p.share >> 3;
  if (off <= near) return x - off;
  if (s.chunks - off <= near) return x - off + s.chunks;
  return x;
}

// walks over the chunks of a CTA
template <int C, int ROWS>
struct Walk {
  long long at, end;                    // next chunk, end of the share
  Seq s;
  int b, tile, c, c_end;                // tile of the sequence; next chunk of it, end of the share's part
  long long tile_start;
  __device__ void init(const Args& a, const Plan& p, int cta) {
    if (p.whole) {
      const bool any = cta < p.tile_base[p.batch];
      b = any ? find(p.tile_base, p.batch, cta) : 0;
      s = sequence<C, ROWS>(a, b);
      at = any ? p.base[b] + (long long)(cta - p.tile_base[b]) * s.chunks : 0;
      end = any ? at + s.chunks : 0;
    } else {
      at = boundary<C, ROWS>(a, p, cta);
      end = boundary<C, ROWS>(a, p, cta + 1);
      b = at < end ? find(p.base, p.batch, at) : 0;
      s = sequence<C, ROWS>(a, b);
    }
  }
  // the next tile, or part of one
  __device__ bool next(const Args& a, const Plan& p) {
    if (at >= end) return false;
    if (at >= p.base[b + 1]) {
      do ++b; while (p.base[b + 1] == p.base[b]);
      s = sequence<C, ROWS>(a, b);
    }
    const long long in = at - p.base[b];
    tile = (int)(in / s.chunks);
    tile_start = p.base[b] + (long long)tile * s.chunks;
    c = (int)(at - tile_start);
    c_end = (int)(end - tile_start < s.chunks ? end - tile_start : s.chunks);
    at = tile_start + c_end;
    return true;
  }
};

// a chunk: keys [start, start + n) of the cache, or nodes
struct Chunk { int start, n; bool tree; };
template <int C>
__device__ inline Chunk chunk_of(const Seq& s, int c) {
  Chunk k;
  k.tree = c >= s.n_pre + s.n_main;
  if (k.tree) { k.start = (c - s.n_pre - s.n_main) * C; k.n = min(C, s.n - k.start); }
  else if (c < s.n_pre) { k.start = c * C; k.n = min(C, s.pre - k.start); }
  else { k.start = s.lo + (c - s.n_pre) * C; k.n = min(C, s.len - k.start); }
  return k;
}

// ---- prefix sums over the sequences, by a block of THREADS
template <int C, int ROWS, int THREADS>
__device__ inline void make_plan(const Args& a, Plan& p, long long* base, int* tile_base, long long* sh) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  long long carry = 0;
  int t_carry = 0, longest = 0;
  for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
    const int b = b0 + threadIdx.x;
    long long units = 0;
    int tiles = 0;
    if (b < a.batch) {
      const Seq s = sequence<C, ROWS>(a, b);
      tiles = s.tiles * a.Hkv;
      units = (long long)tiles * s.chunks;
      if (tiles > 0) longest = max(longest, s.chunks);
    }
    long long x = units;
    int t = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      const int z = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) { x += y; t += z; }
    }
    __syncthreads();
    if (lane == 31) { sh[2 * w] = x; sh[2 * w + 1] = t; }
    __syncthreads();
    long long bx = carry;
    int bt = t_carry;
    for (int k = 0; k < THREADS / 32; ++k) {
      if (k < w) { bx += sh[2 * k]; bt += (int)sh[2 * k + 1]; }
      carry += sh[2 * k];
      t_carry += (int)sh[2 * k + 1];
    }
    if (b < a.batch) { base[b] = bx + x - units; tile_base[b] = bt + t - tiles; }
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  __syncthreads();
  if (lane == 0) sh[w] = longest;
  if (threadIdx.x == 0) { base[a.batch] = carry; tile_base[a.batch] = t_carry; }
  __syncthreads();
  for (int k = 0; k < THREADS / 32; ++k) longest = max(longest, (int)sh[k]);
  p.base = base; p.tile_base = tile_base; p.batch = a.batch;
  p.total = carry;
  p.share = (carry + gridDim.x - 1) / gridDim.x;
  if (p.share < 1) p.share = 1;
  // Few tiles that are short, or all alike: a CTA each.  (Cutting a tile of up to six chunks costs more in parts than it gains.)
  const long long most = p.share + (p.share >> 2) > 6 ? p.share + (p.share >> 2) : 6;
  p.whole = t_carry <= (int)gridDim.x && longest <= most;
}

// CTA `cta` starts a tile that it does not end: how many CTAs share it
template <int C, int ROWS>
__device__ inline int parts_of(const Args& a, const Plan& p, int cta, long long tile_end) {
  int n = 1;
  while (cta + n < (int)gridDim.x && boundary<C, ROWS>(a, p, cta + n) < tile_end) ++n;
  return n;
}

// ---- ancestors of the nodes of a sequence, by `threads` threads that meet at `bar`: reach[i] (zero: not in use), depth[i]
struct Tree {
  uint32_t reach[FM_MAX_TREE_NODES][WORDS];
  short jump[FM_MAX_TREE_NODES];
  short depth[FM_MAX_TREE_NODES];
  int max_depth;
};
template <int THREADS, typename Sync>
__device__ inline void build_tree(Tree& t, const int* parent, int n, int tid, Sync sync) {
  constexpr int PER = FM_MAX_TREE_NODES / THREADS;
  const int words = (n + 31) >> 5;
  sync();                                                    // the last tree is no longer read
  if (tid == 0) t.max_depth = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = k * THREADS + tid;
    if (i < n) {
      const int p = parent[i];
      t.jump[i] = (short)(p == -1 ? -1 : (p >= 0 && p < i ? p : -2));
      for (int w = 0; w < words; ++w) t.reach[i][w] = w == (i >> 5) ? 1u << (i & 31) : 0u;
    }
  }
  sync();
  for (int span = 1; span < n; span <<= 1) {
    uint32_t up[PER][WORDS];
    int to[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = k * THREADS + tid;
      to[k] = -3;
      if (i < n && t.jump[i] >= 0) {
        const int j = t.jump[i];
        to[k] = t.jump[j];
#pragma unroll
        for (int w = 0; w < WORDS; ++w) up[k][w] = w < words ? t.reach[j][w] : 0u;
      }
    }
    sync();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int i = k * THREADS + tid;
      if (to[k] != -3) {
#pragma unroll
        for (int w = 0; w < WORDS; ++w) if (w < words) t.reach[i][w] |= up[k][w];
        t.jump[i] = (short)to[k];
      }
    }
    sync();
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = k * THREADS + tid;
    if (i < n) {
      int d = -1;
      for (int w = 0; w < words; ++w) {
        if (t.jump[i] == -2) t.reach[i][w] = 0u;
        d += __popc(t.reach[i][w]);
      }
      t.depth[i] = (short)d;
      atomicMax(&t.max_depth, d);
    }
  }
  sync();
}

// ------------------------------------------------------------------------------------------
// sixteen query rows a tile, warp-level MMAs
// ------------------------------------------------------------------------------------------
template <int DH>
struct Rows16 {
  static constexpr int ROWS = 16, C = DH == 64 ? 128 : 64, NW = 4, KPW = C / NW, STAGES = 4;
  static constexpr int TILE = C * DH * 2, STAGE = 2 * TILE, RING = STAGES * STAGE;
  static constexpr int STATES = NW * 16 * (DH + 2) * 4;
  static constexpr int THREADS = 256;                        // four multiplying, four loading warps
  static constexpr int FIXED = RING + STATES + (int)sizeof(Tree) + 1024 + 256;
  static int bytes(int batch) { return FIXED + (batch + 1) * 12 + 16; }
};

template <typename T, int DH>
__global__ void __launch_bounds__(256, 1) rows16_kernel(const __grid_constant__ Args a) {
  using CF = Rows16<DH>;
  constexpr int C = CF::C, NW = CF::NW, KPW = CF::KPW, KS = DH / 16, KB = KPW / 16, NT = KPW / 8, ST = CF::STAGES;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* pw = reinterpret_cast<float*>(sm + CF::RING);       // [NW][16][DH] outputs
  float* ml = pw + NW * 16 * DH;                             // [NW][16][2] maxima and sums
  Tree& tree = *reinterpret_cast<Tree*>(sm + CF::RING + CF::STATES);
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + CF::RING + CF::STATES + ((sizeof(Tree) + 7) & ~size_t(7)));
  uint64_t* empty = full + ST;
  long long* s_sh = reinterpret_cast<long long*>(empty + ST);              // [16]
  long long* s_base = s_sh + 16;
  int* s_tile_base = reinterpret_cast<int*>(s_base + a.batch + 1);
  __shared__ int s_fail;
  const int warp = (int)ptx::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  ptx::grid_dep_launch();
  if (threadIdx.x == 0) {
    s_fail = 0;
    for (int i = 0; i < ST; ++i) { ptx::mbar_init(full + i, 128); ptx::mbar_init(empty + i, NW); }
    ptx::fence_mbar_init();
  }
  Plan plan;
  make_plan<C, 16, CF::THREADS>(a, plan, s_base, s_tile_base, s_sh);
  Walk<C, 16> w;
  w.init(a, plan, blockIdx.x);
  __syncthreads();

  if (warp >= NW) {
    // ---- loading: a thread brings piece `piece` of rows r0, r0 + STEP, ...
    constexpr int PIECES = DH / 8, STEP = 128 / PIECES, RPT = C / STEP;
    const int t = threadIdx.x - NW * 32, piece = t % PIECES, row0 = t / PIECES;
    const uint32_t half_off = (uint32_t)(piece >> 3) * C * 128;
    const T *kc = reinterpret_cast<const T*>(a.k) + piece * 8, *vc = reinterpret_cast<const T*>(a.v) + piece * 8;
    const T *kn = static_cast<const T*>(a.k_new) + piece * 8, *vn = static_cast<const T*>(a.v_new) + piece * 8;
    Chunk cur{}, nxt{};
    int ids[RPT], ids2[RPT];                                 // page ids of the thread's rows (-1: nothing there)
    int hk = 0, hk2 = 0, r0 = 0, r02 = 0, c = 0;
    bool more = w.next(a, plan);
    auto fetch = [&](const Chunk& k, int (&id)[RPT]) {
      if (k.tree) return;
      const int* table = a.table + (int64_t)w.s.seq * a.max_pages;
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const int r = row0 + i * STEP;
        id[i] = r < k.n ? __ldg(table + a.page_div(k.start + r)) : -1;
      }
    };
    auto take = [&](Chunk& k, int& h, int& r) {              // the chunk at the walk's place
      k = chunk_of<C>(w.s, c);
      h = w.tile / w.s.tiles;
      r = w.s.r0;
    };
    if (more) { c = w.c; take(cur, hk, r0); fetch(cur, ids); }
    for (int i = 0; more; ++i) {
      // the next chunk, and its page ids
      bool more2 = true;
      if (++c >= w.c_end) { more2 = w.next(a, plan); c = w.c; }
      if (more2) { take(nxt, hk2, r02); fetch(nxt, ids2); }
      const int st = i % ST;
      if (i >= ST && !__all_sync(0xffffffffu, ptx::mbar_wait(empty + st, ((i / ST) - 1) & 1))) { s_fail = 1; break; }
      const uint32_t Ks = ptx::smem_u32(sm + st * CF::STAGE) + half_off, Vs = Ks + CF::TILE;
#pragma unroll
      for (int j = 0; j < RPT; ++j) {
        const int r = row0 + j * STEP;
        bool there = r < cur.n;
        int64_t at = 0;
        const T *ks = kc, *vs = vc;
        if (cur.tree) {
          if (there) at = (int64_t)(r0 + cur.start + r) * a.new_row + hk * DH;
          ks = kn; vs = vn;
        } else if (there) {
          const int s = cur.start + r, id = ids[j];
          if (id < 0 || id >= a.n_pages) {
            there = false;
            if (a.status != nullptr) atomicMin(a.status, FM_ERR_INVALID_ARG);
          } else {
            at = id * a.page + hk * a.head + (int64_t)(s - a.page_div(s) * a.page_div.d) * a.slot;
          }
        }
        const uint32_t to = ptx::swz128(r, piece & 7);
        cp16(Ks + to, ks + at, there);
        cp16(Vs + to, vs + at, there);
      }
      cp_arrive(full + st);
      more = more2;
      cur = nxt; hk = hk2; r0 = r02;
#pragma unroll
      for (int j = 0; j < RPT; ++j) ids[j] = ids2[j];
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    // ---- multiplying
    auto sync = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
    int tree_of = -1, it = 0;
    if (threadIdx.x == 0) a.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
    while (w.next(a, plan)) {
      const Seq& s = w.s;
      const int hk = w.tile / s.tiles, mt = w.tile - hk * s.tiles, M = s.n * a.G;
      if (tree_of != w.b) { build_tree<128>(tree, a.parent + s.r0, s.n, threadIdx.x, sync); tree_of = w.b; }
      const bool whole = w.c == 0 && w.c_end == s.chunks;
      if (threadIdx.x == 0 && w.c == 0 && !whole)
        a.desc[blockIdx.x] = make_int4(w.b, hk, mt, parts_of<C, 16>(a, plan, blockIdx.x, w.tile_start + s.chunks));
      uint32_t qa[KS][4];
      int node[2];                                           // the rows' nodes, -1: behind the last
#pragma unroll
      for (int hr = 0; hr < 2; ++hr) {
        const int idx = mt * 16 + g + hr * 8;
        const bool ok = idx < M;
        const int i = ok ? idx / a.G : 0, gh = ok ? idx - i * a.G : 0;
        node[hr] = ok ? i : -1;
        const T* qp = static_cast<const T*>(a.q) + (int64_t)(s.r0 + i) * a.q_row + (hk * a.G + gh) * DH;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qa[ks][hr] = ok ? __ldg(reinterpret_cast<const unsigned int*>(qp + ks * 16 + 2 * t4)) : 0u;
          qa[ks][2 + hr] = ok ? __ldg(reinterpret_cast<const unsigned int*>(qp + ks * 16 + 8 + 2 * t4)) : 0u;
        }
      }
      // first cached position behind the prefix that a row sees
      int depth[2], low[2];
#pragma unroll
      for (int hr = 0; hr < 2; ++hr) {
        depth[hr] = node[hr] >= 0 ? tree.depth[node[hr]] : 0;
        low[hr] = a.window > 0 ? s.len + depth[hr] - a.window + 1 : 0;
      }
      const int low_all = a.window > 0 ? s.len + tree.max_depth - a.window + 1 : 0;
      float o[DH / 8][4];
      float mrun[2] = {-INFINITY, -INFINITY}, lrun[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
      bool gave_up = false;
      for (int c = w.c; c < w.c_end; ++c, ++it) {
        const Chunk ck = chunk_of<C>(s, c);
        const int st = it % ST;
        const bool uneven = ck.tree || (a.window > 0 && ck.start + ck.n > a.n_prefix && ck.start < low_all);   // rows differ in what they see
        const bool all_vis = !uneven && ck.n == C;
        if (!__all_sync(0xffffffffu, ptx::mbar_wait(full + st, (it / ST) & 1))) { gave_up = true; break; }
        const uint32_t Ks_u = ptx::smem_u32(sm + st * CF::STAGE), Vs_u = Ks_u + CF::TILE;
        uint32_t kf[KB][KS][4], vf[KB][DH / 16][4];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const int key = warp * KPW + kb * 16 + (lane & 7) + (lane >> 4) * 8;
            const int ch = ks * 2 + ((lane >> 3) & 1);
            ptx::ldmatrix_x4(kf[kb][ks][0], kf[kb][ks][1], kf[kb][ks][2], kf[kb][ks][3], Ks_u + (ch >> 3) * C * 128 + ptx::swz128(key, ch & 7));
          }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int dp = 0; dp < DH / 16; ++dp) {
            const int key = warp * KPW + kb * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
            const int ch = dp * 2 + (lane >> 4);
            ptx::ldmatrix_x4_trans(vf[kb][dp][0], vf[kb][dp][1], vf[kb][dp][2], vf[kb][dp][3], Vs_u + (ch >> 3) * C * 128 + ptx::swz128(key, ch & 7));
          }
        float sc[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            mma16816(sc[2 * kb], qa[ks], kf[kb][ks][0], kf[kb][ks][1], T());
            mma16816(sc[2 * kb + 1], qa[ks], kf[kb][ks][2], kf[kb][ks][3], T());
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nt][e] *= a.scale_log2;
        bool bad = false;
        if (!all_vis) {
          // keys of this thread: n-tile nt, element e -> nt * 8 + 2 * t4 + e of the warp's slice
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int k = warp * KPW + nt * 8 + 2 * t4 + e, at = ck.start + k;
#pragma unroll
              for (int hr = 0; hr < 2; ++hr) {
                bool vis = k < ck.n && node[hr] >= 0;
                if (vis && ck.tree) vis = ((tree.reach[node[hr]][at >> 5] >> (at & 31)) & 1u) && (a.window == 0 || depth[hr] - tree.depth[at] < a.window);
                else if (vis && uneven) vis = at < a.n_prefix || at >= low[hr];
                if (!vis) sc[nt][hr * 2 + e] = -INFINITY;
              }
            }
          if (uneven) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int dp = 0; dp < DH / 16; ++dp)
#pragma unroll
                for (int j = 0; j < 4; ++j) vf[kb][dp][j] = finite_part<T>(vf[kb][dp][j], bad);
          }
        }
        float scale[2], base[2];
#pragma unroll
        for (int hr = 0; hr < 2; ++hr) {
          float mx = -INFINITY;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mx = fmaxf(mx, fmaxf(sc[nt][hr * 2], sc[nt][hr * 2 + 1]));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          const float mnew = fmaxf(mrun[hr], mx);
          base[hr] = mnew == -INFINITY ? 0.f : mnew;
          scale[hr] = mnew == mrun[hr] ? 1.f : ex2(mrun[hr] - base[hr]);
          mrun[hr] = mnew;
        }
        float ls[2] = {0.f, 0.f};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[nt][e] = ex2(sc[nt][e] - base[e >> 1]);
            ls[e >> 1] += sc[nt][e];
          }
        lrun[0] = lrun[0] * scale[0] + ls[0];
        lrun[1] = lrun[1] * scale[1] + ls[1];
        if (__any_sync(0xffffffffu, scale[0] != 1.f || scale[1] != 1.f)) {
#pragma unroll
          for (int i = 0; i < DH / 8; ++i) {
            o[i][0] *= scale[0]; o[i][1] *= scale[0];
            o[i][2] *= scale[1]; o[i][3] *= scale[1];
          }
        }
        // P is rounded to the cache's type for the tensor cores: half a step of it per term, as much again as the rounding of
        // the output itself; the sums are those of the unrounded values
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          uint32_t pa[4];
          pa[0] = pack(sc[2 * kb][0], sc[2 * kb][1], T());
          pa[1] = pack(sc[2 * kb][2], sc[2 * kb][3], T());
          pa[2] = pack(sc[2 * kb + 1][0], sc[2 * kb + 1][1], T());
          pa[3] = pack(sc[2 * kb + 1][2], sc[2 * kb + 1][3], T());
#pragma unroll
          for (int dp = 0; dp < DH / 16; ++dp) {
            mma16816(o[2 * dp], pa, vf[kb][dp][0], vf[kb][dp][1], T());
            mma16816(o[2 * dp + 1], pa, vf[kb][dp][2], vf[kb][dp][3], T());
          }
        }
        if (__any_sync(0xffffffffu, bad)) {
          // values that are not finite: key by key, for the rows that see the key (p > 0)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            for (int k = 0; k < 8; ++k) {
              const int key = warp * KPW + nt * 8 + k, src = (lane & ~3) | (k >> 1);
              const float p0 = __shfl_sync(0xffffffffu, (k & 1) ? sc[nt][1] : sc[nt][0], src);
              const float p1 = __shfl_sync(0xffffffffu, (k & 1) ? sc[nt][3] : sc[nt][2], src);
#pragma unroll
              for (int i = 0; i < DH / 8; ++i) {
                const int col = i * 8 + 2 * t4;
                const uint32_t raw = *reinterpret_cast<const uint32_t*>(sm + st * CF::STAGE + CF::TILE + (col >> 6) * C * 128 +
                                                                       ptx::swz128(key, (col & 63) >> 3) + (col & 7) * 2);
                const float2 v = unpack(raw, T());
                if (!(fabsf(v.x) < INFINITY)) { if (p0 != 0.f) o[i][0] += p0 * v.x; if (p1 != 0.f) o[i][2] += p1 * v.x; }
                if (!(fabsf(v.y) < INFINITY)) { if (p0 != 0.f) o[i][1] += p0 * v.y; if (p1 != 0.f) o[i][3] += p1 * v.y; }
              }
            }
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(empty + st);
      }
      if (gave_up) { s_fail = 1; }
#pragma unroll
      for (int hr = 0; hr < 2; ++hr) {
        lrun[hr] += __shfl_xor_sync(0xffffffffu, lrun[hr], 1);
        lrun[hr] += __shfl_xor_sync(0xffffffffu, lrun[hr], 2);
      }
      // ---- the warps' states, merged in warp order
      float* mine = pw + warp * 16 * DH;
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) {
        *reinterpret_cast<float2*>(mine + g * DH + i * 8 + 2 * t4) = make_float2(o[i][0], o[i][1]);
        *reinterpret_cast<float2*>(mine + (g + 8) * DH + i * 8 + 2 * t4) = make_float2(o[i][2], o[i][3]);
      }
      if (t4 == 0) {
        *reinterpret_cast<float2*>(ml + (warp * 16 + g) * 2) = make_float2(mrun[0], lrun[0]);
        *reinterpret_cast<float2*>(ml + (warp * 16 + g + 8) * 2) = make_float2(mrun[1], lrun[1]);
      }
      sync();
      if (*reinterpret_cast<volatile int*>(&s_fail)) break;  // (every warp has set its word in front of the barrier: all leave)
      const int rows_here = min(16, M - mt * 16);
      float* part = a.part + (size_t)(blockIdx.x * 2 + (w.c == 0 ? 1 : 0)) * 16 * (DH + 2);
      for (int e = threadIdx.x; e < rows_here * (DH / 2); e += 128) {
        const int i = e / (DH / 2), col = 2 * (e - i * (DH / 2)), idx = mt * 16 + i, nd = idx / a.G, gh = idx - nd * a.G;
        const bool live = tree.reach[nd][nd >> 5] != 0u;
        float2 stt[NW];
        float mm = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) { stt[k] = *reinterpret_cast<const float2*>(ml + (k * 16 + i) * 2); mm = fmaxf(mm, stt[k].x); }
#pragma unroll
        for (int k = 0; k < NW; ++k) {
          const float f = stt[k].x == -INFINITY ? (stt[k].y == stt[k].y ? 0.f : 1.f) : ex2(stt[k].x - mm);
          const float2 v = *reinterpret_cast<const float2*>(pw + (k * 16 + i) * DH + col);
          if (f != 0.f) { l += f * stt[k].y; o0 += f * v.x; o1 += f * v.y; }
        }
        if (!live) { mm = -INFINITY; l = o0 = o1 = 0.f; }
        if (whole) {
          const float inv = live ? 1.f / l : 0.f;
          *reinterpret_cast<uint32_t*>(static_cast<T*>(a.out) + (int64_t)(s.r0 + nd) * a.out_row + (hk * a.G + gh) * DH + col) = pack(o0 * inv, o1 * inv, T());
          if (col == 0 && a.lse != nullptr) a.lse[(int64_t)(s.r0 + nd) * a.H + hk * a.G + gh] = live ? (mm + log2f(l)) * 0.6931471805599453f : -INFINITY;
        } else {
          float* row = part + (size_t)i * (DH + 2);
          *reinterpret_cast<float2*>(row + col) = make_float2(o0, o1);
          if (col == 0) *reinterpret_cast<float2*>(row + DH) = make_float2(mm, l);
        }
      }
      sync();                                                // the states have been read
    }
  }
  __syncthreads();
  if (s_fail) {                                              // a bounded wait gave up: report
    if (threadIdx.x == 0 && a.status != nullptr) atomicMin(a.status, FM_ERR_TIMEOUT);
  }
}

// ---- parts of the tiles that were cut, merged in order: grid (CTAS, ROWS / 4), two warps a row
template <typename T, int DH, int ROWS>
__global__ void __launch_bounds__(256) merge_kernel(const __grid_constant__ Args a) {
  constexpr int CL = DH / 32, GS = ROWS * (DH + 2);
  __shared__ float s_o[4][DH];
  __shared__ float2 s_ml[4];
  ptx::grid_dep_wait();
  const int4 d = __ldcg(a.desc + blockIdx.x);
  if (d.w < 2) return;
  const int r0 = a.row_off[d.x], n = min(a.row_off[d.x + 1] - r0, a.max_nodes), M = n * a.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = warp & 3, half = warp >> 2, i = blockIdx.y * 4 + r, idx = d.z * ROWS + i;
  if (d.z * ROWS + (int)blockIdx.y * 4 >= M) return;
  const bool there = idx < M;
  float m = -INFINITY, l = 0.f, o[CL];
#pragma unroll
  for (int j = 0; j < CL; ++j) o[j] = 0.f;
  auto add = [&](float m2, float l2, const float (&o2)[CL]) {
    if (m2 == -INFINITY && l2 == 0.f) return;
    const float mn = fmaxf(m, m2), f1 = m == -INFINITY && l == 0.f ? 0.f : ex2(m - mn), f2 = m2 == -INFINITY ? 1.f : ex2(m2 - mn);
    l = (f1 == 0.f ? 0.f : l * f1) + l2 * f2;
#pragma unroll
    for (int j = 0; j < CL; ++j) o[j] = (f1 == 0.f ? 0.f : o[j] * f1) + (f2 == 0.f ? 0.f : o2[j] * f2);
    m = mn;
  };
  if (there) {
    constexpr int U = 4;
    for (int k0 = half; k0 < d.w; k0 += 2 * U) {
      float2 ml[U];
      float v[U][CL];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = k0 + 2 * u;
        if (k >= d.w) continue;
        const float* row = a.part + ((size_t)(blockIdx.x + k) * 2 + (k == 0 ? 1 : 0)) * GS + (size_t)i * (DH + 2);
        ml[u] = __ldcg(reinterpret_cast<const float2*>(row + DH));
#pragma unroll
        for (int j = 0; j < CL; ++j) v[u][j] = __ldcg(row + lane + 32 * j);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (k0 + 2 * u < d.w) add(ml[u].x, ml[u].y, v[u]);
    }
  }
  if (half == 1) {
#pragma unroll
    for (int j = 0; j < CL; ++j) s_o[r][lane + 32 * j] = o[j];
    if (lane == 0) s_ml[r] = make_float2(m, l);
  }
  __syncthreads();
  if (half == 1 || !there) return;
  float o2[CL];
#pragma unroll
  for (int j = 0; j < CL; ++j) o2[j] = s_o[r][lane + 32 * j];
  add(s_ml[r].x, s_ml[r].y, o2);
  const int nd = idx / a.G, gh = idx - nd * a.G, h = d.y * a.G + gh;
  const bool live = !(m == -INFINITY && l == 0.f);           // (a node in use sees itself)
  const float inv = live ? 1.f / l : 0.f;
  T* out = static_cast<T*>(a.out) + (int64_t)(r0 + nd) * a.out_row + (int64_t)h * DH;
#pragma unroll
  for (int j = 0; j < CL; ++j) {
    const uint32_t v = pack(o[j] * inv, 0.f, T());
    reinterpret_cast<unsigned short*>(out)[lane + 32 * j] = (unsigned short)v;
  }
  if (lane == 0 && a.lse != nullptr) a.lse[(int64_t)(r0 + nd) * a.H + h] = live ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// ------------------------------------------------------------------------------------------
// the longest confirmed path: a warp per tree, eight nodes a lane
// ------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(128) accept_kernel(const int* tokens, const int* parent, const int* row_off, const int* predicted, int batch,
                                                     int* path, int path_stride, int* n_acc, int* next_tok) {
  constexpr int PER = FM_MAX_TREE_NODES / 32;
  const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= batch) return;
  const int r0 = row_off[b], n = r0 < 0 ? 0 : min(min(row_off[b + 1] - r0, FM_MAX_TREE_NODES), path_stride);
  int par[PER], tok[PER], pre[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = k * 32 + lane;
    par[k] = i < n ? parent[r0 + i] : -2;
    tok[k] = i < n ? tokens[r0 + i] : 0;
    pre[k] = i < n ? predicted[r0 + i] : 0;
  }
  int cur = n > 0 && __shfl_sync(0xffffffffu, par[0], 0) == -1 ? 0 : -1, at = 0, want = -1;
  while (cur >= 0) {                                         // (every step goes to a later node)
    if (lane == 0) path[(int64_t)b * path_stride + at] = cur;
    ++at;
    int mine = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) if ((cur >> 5) == k) mine = pre[k];
    want = __shfl_sync(0xffffffffu, mine, cur & 31);
    int next = -1;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const unsigned hit = __ballot_sync(0xffffffffu, par[k] == cur && tok[k] == want && k * 32 + lane > cur);
      if (next < 0 && hit != 0) next = k * 32 + __ffs(hit) - 1;
    }
    cur = next;
  }
  for (int j = at + lane; j < path_stride; j += 32) path[(int64_t)b * path_stride + j] = -1;
  if (lane == 0) { n_acc[b] = at; next_tok[b] = at > 0 ? want : -1; }
}

}  // namespace tr
