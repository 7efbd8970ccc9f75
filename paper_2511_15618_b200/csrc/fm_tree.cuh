// Attention of trees of drafted tokens over a paged cache, and the walk that accepts a path.
//
// A tile is what shares keys: the query rows (nodes x heads of the group) of one sequence and kv-head, 16 or 256 of them.  Its keys
// come in chunks of C: conditioning slots, the window's slots (or all cached ones), the nodes.  The launch is one CTA
// per SM whatever the lengths: the chunks of all tiles, one tile after the other, are cut into equal shares (their total is
// known on the device alone), so ragged batches are balanced without the host.  A cut falls inside a tile at most once per CTA; the
// parts of a cut tile go to a scratch buffer and a second small launch merges them in order.
// Loading: a page's slots (or a chunk's, or as many as fit evenly into both) of a head are one TMA box, swizzled for the
// multiplication; warps of their own request chunks ahead, through a ring of stages.  Smaller boxes than a lane each can bring
// (pages that are no multiple of 4 slots; of 2, chunks of 64), and the nodes' rows, are copied 16 bytes a thread (cp.async) into the same layout.
// 64 sequences of 100 to 8000 positions, 8 kv-heads of 128: pages of 64 and 16 103 us, 8 130, 100 133 (234 when copied), 4 145, 3 289 (copied).
// Ancestors: reach[i], a bit per node, by pointer doubling over the parents (log2 of the depth rounds).
// Values a row does not see have no effect on it: scores are replaced by -inf; values that are not finite in chunks
// where some row does not see all keys are taken out of the product and added to the rows that do see them.
#pragma once
#include <cuda_fp16.h>

#include "fm_common.cuh"
#include "fm_gemm_tc.cuh"
#include "fm_ptx.cuh"
#include "../../include/flashmesh.h"

namespace tr {

constexpr int SMS = 148;                // of a B200: one CTA each; the workspace is laid out for them
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
  float* part;                          // [CTAs * 2][ROWS][DH + 2]
  int4* desc;                           // [CTAs]: sequence, kv-head, tile, parts of the tile that starts here and is cut
  Div page_div, g_div;                  // by the slots of a page, by the heads of a group
  int n_pages, max_pages, max_seqs, batch, H, Hkv, G, max_nodes, max_len, window, n_prefix;
  float scale_log2;
  int ring;                             // 0, or: positions behind the prefix wrap around after so many slots (one page per sequence)
  int lo_off;                           // 0, or: rows are [hi | lo] bfloat16 terms, lo so many elements behind hi
  int tma, box_rows;                    // the page size suits boxes, of so many slots
  int n_rows, fill;                     // rows that there are (0: not said); what rows of no tree get: FM_FILL_*
  alignas(64) CUtensorMap map_k, map_v; // the layer's pool as [pages][heads][slots][head_dim], box 64 features x box_rows slots
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

// the larger of the halves' magnitudes (their bits without the sign), half by half: those of what is not finite stay on top
template <typename T>
__device__ inline uint32_t largest(uint32_t m, uint32_t v) { return __vmaxu2(m, v & 0x7fff7fffu); }

// a value that the rounding of a pair to T lost, as a pair of bfloat16 (rows of two terms)
__device__ inline uint32_t pack_rest(float x, float y, uint32_t hi) {
  const float2 h = unpack(hi, bf16());
  return ptx::pack_bf16(__fsub_rn(x, h.x), __fsub_rn(y, h.y));
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

// Exponentials are taken to a reference so many powers of two below the row's maximum; sums and outputs carry the same factor.  Half
// has no number between 0 and 2^-24: weights of an unshifted softmax below 2^-25 would vanish from the product with the values
// and those below 2^-14 lose bits, and in a long cache all of a row but its sink can be such.  A shift of 14 keeps weights down to 2^-28 of
// the largest at full precision and 2^-39 at all (2^14 times a value fits fp32 sums).  bfloat16 has fp32's exponents.
template <typename T> constexpr float SHIFT = __is_same(T, bf16) ? 0.f : 14.f;

// ---- what a sequence asks for
struct Seq {
  int r0, n, len, seq;                  // first row, nodes, cached positions, its row of the table
  int pre, lo;                          // slots [0, pre) and [lo, len) are loaded; both ranges start at a multiple of C
  int n_pre, n_main, chunks, tiles;     // chunks of the two ranges, all chunks, query tiles per kv-head
};
__device__ inline int4 read_sequence(const Args& a, int b) {                   // (r0, n, len, seq) from the caller's arrays; n -1: not rows that there are
  const int r0 = a.row_off[b], end = a.row_off[b + 1], seq = a.seqs != nullptr ? a.seqs[b] : b;
  const int len = seq >= 0 && seq < a.max_seqs ? max(0, min(a.lens[seq], a.max_len)) : 0;
  return make_int4(r0, r0 < 0 || end < r0 || (a.n_rows > 0 && end > a.n_rows) ? -1 : min(end - r0, a.max_nodes), len, seq);
}
template <int C, int ROWS>
__device__ inline Seq sequence(const Args& a, int4 v) {
  Seq s;
  s.r0 = v.x; s.n = v.y; s.len = v.z; s.seq = v.w;
  s.pre = min(a.n_prefix, s.len);
  s.lo = a.window > 0 ? max(s.pre, s.len - a.window + 1) : 0;
  s.lo = min(s.lo, s.len) / C * C;
  if (s.lo < (s.pre + C - 1) / C * C) { s.pre = 0; s.lo = 0; }                 // one range
  s.n_pre = (s.pre + C - 1) / C;
  s.n_main = (s.len - s.lo + C - 1) / C;
  s.chunks = s.n_pre + s.n_main + (s.n + C - 1) / C;
  s.tiles = (s.n * a.G + ROWS - 1) / ROWS;
  return s;
}

// ---- the cut of all chunks into shares.  A tile counts OVER chunks more than it has: what starting and ending it takes.  (2, 4, 6, 8:
// geometric means over 17 ragged and even batches of 97.5, 95.4, 94.1 and 95.3 us.)  A cut of up to NEAR chunks off the border
// of a tile moves there; an eighth of a share in place of 3 chunks left some CTAs a quarter more than others (202 us for then 179
// at 64 sequences of 4000 positions, 8 kv-heads of 128).
constexpr int OVER = 6, NEAR = 3;
struct Plan {
  const long long* base;                // [batch + 1] units in front of a sequence's
  const int* tile_base;                 // [batch + 1] tiles in front of a sequence's
  const int4* info;                     // [batch]
  int batch;
  long long total, share;
  bool whole;                           // CTA i takes tile i: nothing is cut
  bool left;                            // some tree has rows that take no part
};
// last sequence whose first unit (tile) is not behind x, and that has any
template <typename V>
__device__ inline int find(const V* base, int batch, long long x) {
  int lo = 0, hi = batch;                                    // base[lo] <= x < base[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((long long)base[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}
// first unit of CTA i's share.  A cut close to the border of a tile moves there: the tile stays whole.
template <int C, int ROWS>
__device__ inline long long boundary(const Args& a, const Plan& p, int i) {
  const long long x = p.share * i;
  if (i <= 0) return 0;
  if (x >= p.total) return p.total;
  const int b = find(p.base, p.batch, x), units = sequence<C, ROWS>(a, p.info[b]).chunks + OVER;
  const int off = (int)((x - p.base[b]) % units);
  const long long near = (p.share >> 3) < NEAR ? (p.share >> 3) : NEAR;
  if (off <= near + OVER) return x - off;
  if (units - off <= near) return x - off + units;
  return x;
}

// walks over the chunks of a CTA
template <int C, int ROWS>
struct Walk {
  long long at, end;                    // next unit, end of the share
  Seq s;
  int b, hk, mt, c, c_end;              // sequence, kv-head and tile of it; next chunk of it, end of the share's part
  long long tile_start;
  bool inside;                          // next() has been called in this sequence
  __device__ void init(const Args& a, const Plan& p, int cta) {
    if (p.whole) {
      const bool any = cta < p.tile_base[p.batch];
      b = any ? find(p.tile_base, p.batch, cta) : 0;
      s = sequence<C, ROWS>(a, p.info[b]);
      at = any ? p.base[b] + (long long)(cta - p.tile_base[b]) * (s.chunks + OVER) : 0;
      end = any ? at + s.chunks + OVER : 0;
    } else {
      at = boundary<C, ROWS>(a, p, cta);
      end = boundary<C, ROWS>(a, p, cta + 1);
      b = at < end ? find(p.base, p.batch, at) : 0;
      s = sequence<C, ROWS>(a, p.info[b]);
    }
    inside = false;
  }
  // the next tile, or part of one
  __device__ bool next(const Args& a, const Plan& p) {
    if (at >= end) return false;
    if (at >= p.base[b + 1]) {
      do ++b; while (p.base[b + 1] == p.base[b]);
      s = sequence<C, ROWS>(a, p.info[b]);
      inside = false;
    }
    const int units = s.chunks + OVER;
    if (inside) {
      if (++mt == s.tiles) { mt = 0; ++hk; }
      tile_start = at;
    } else {
      const long long in = at - p.base[b];
      const int tile = (in >> 31) == 0 ? (int)in / units : (int)(in / units);
      hk = tile / s.tiles;
      mt = tile - hk * s.tiles;
      tile_start = p.base[b] + (long long)tile * units;
      inside = true;
    }
    c = max(0, (int)(at - tile_start) - OVER);               // (cuts lie behind the first OVER units or in front of them)
    c_end = (int)(end - tile_start < units ? end - tile_start : units) - OVER;
    at = tile_start + OVER + c_end;
    return true;
  }
  __device__ bool starts() const { return c == 0; }
  __device__ bool ends() const { return c_end == s.chunks; }
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

// where position-slot `slot` of a sequence lies in its pages
__device__ inline int place_of(const Args& a, int slot) { return a.ring > 0 && slot >= a.n_prefix ? a.n_prefix + (slot - a.n_prefix) % a.ring : slot; }
// is the chunk brought as boxes?  (not where it runs over the end of a ring)
__device__ inline bool boxed(const Args& a, const Chunk& k) {
  if (!a.tma || k.tree) return false;
  if (a.ring == 0) return true;
  const int last = k.start + k.n - 1;
  return last < a.n_prefix || place_of(a, last) - place_of(a, k.start) == k.n - 1;
}

// ---- prefix sums over the sequences, by a block of THREADS
template <int C, int ROWS, int THREADS>
__device__ inline void make_plan(const Args& a, Plan& p, int4* info, long long* base, int* tile_base, long long* sh) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  long long carry = 0;
  int t_carry = 0, longest = 0, left = 0;
  for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
    const int b = b0 + threadIdx.x;
    long long units = 0;
    int tiles = 0;
    if (b < a.batch) {
      int4 v = read_sequence(a, b);
      const bool none = v.y < 0, cut = !none && a.row_off[b + 1] - v.x > v.y;        // (cut: more nodes than the caller said)
      if (none) v.y = 0;
      info[b] = v;
      left |= none || cut;
      if ((none || cut) && blockIdx.x == 0 && a.status != nullptr) atomicMin(a.status, none ? FM_ERR_INVALID_ARG : FM_ERR_CAPACITY);
      const Seq s = sequence<C, ROWS>(a, v);
      tiles = s.tiles * a.Hkv;
      units = (long long)tiles * (s.chunks + OVER);
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
    for (int k = 0; k < (THREADS + 31) / 32; ++k) {
      if (k < w) { bx += sh[2 * k]; bt += (int)sh[2 * k + 1]; }
      carry += sh[2 * k];
      t_carry += (int)sh[2 * k + 1];
    }
    if (b < a.batch) { base[b] = bx + x - units; tile_base[b] = bt + t - tiles; }
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  p.left = __syncthreads_or(left) != 0;
  if (lane == 0) sh[w] = longest;
  if (threadIdx.x == 0) { base[a.batch] = carry; tile_base[a.batch] = t_carry; }
  __syncthreads();
  for (int k = 0; k < THREADS / 32; ++k) longest = max(longest, (int)sh[k]);
  p.base = base; p.tile_base = tile_base; p.info = info; p.batch = a.batch;
  p.total = carry;
  p.share = (carry + gridDim.x - 1) / gridDim.x;
  if (p.share <= 2 * OVER) p.share = 2 * OVER + 1;           // (a cut inside a tile then leaves chunks on both sides)
  // Few tiles that are short, or all alike: a CTA each.  (Cutting a tile of up to eight chunks costs more in parts than it gains.)
  const long long most = p.share + (p.share >> 2) > 8 ? p.share + (p.share >> 2) : 8;
  p.whole = t_carry <= (int)gridDim.x && longest <= most;
}
// Rows of no tree: in front of the first and behind the last one, and nodes that take no part.  Output 0, lse -inf.
template <int DH>
__device__ inline void fill_row(const Args& a, int64_t r) {  // by all threads
  if (a.fill & FM_FILL_OUT) {
    uint4* at = reinterpret_cast<uint4*>(static_cast<unsigned short*>(a.out) + r * a.out_row);
    for (int i = threadIdx.x; i < a.H * (DH / 8); i += blockDim.x) at[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  if (a.lse != nullptr && (a.fill & FM_FILL_LSE))
    for (int i = threadIdx.x; i < a.H; i += blockDim.x) a.lse[r * a.H + i] = -INFINITY;
}
// first row of the first tree, and of none behind the last (read before the plan is made: its loads hide these)
__device__ inline int2 ends_of(const Args& a) { return a.fill != 0 ? make_int2(a.row_off[0], a.row_off[a.batch]) : make_int2(0, 0); }
__device__ inline bool to_fill(const Args& a, const Plan& p, int2 ends) { return a.fill != 0 && (p.left || ends.x > 0 || ends.y < a.n_rows); }
template <int DH>
__device__ inline void fill(const Args& a, const Plan& p, int2 ends) {
  if (!p.left) {                                             // (the trees' rows are neighbours and inside the rows that there are)
    const int first = ends.x, last = ends.y;
    for (int64_t r = blockIdx.x; r < first; r += gridDim.x) fill_row<DH>(a, r);
    for (int64_t r = (int64_t)last + blockIdx.x; r < a.n_rows; r += gridDim.x) fill_row<DH>(a, r);
    return;
  }
  // Some are cut short or none (an error of the caller's): row by row, is it a tree's?
  for (int64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    int in = 0;
    for (int b = threadIdx.x; b < a.batch; b += blockDim.x) in |= r >= p.info[b].x && r - p.info[b].x < p.info[b].y;
    if (!__syncthreads_or(in)) fill_row<DH>(a, r);
  }
}
__host__ __device__ constexpr int plan_bytes(int batch) { return 16 * batch + 12 * (batch + 1) + 24; }

// CTA `cta` starts a tile that it does not end: how many CTAs share it
template <int C, int ROWS>
__device__ inline int parts_of(const Args& a, const Plan& p, int cta, long long tile_end) {
  int n = 1;
  while (cta + n < (int)gridDim.x && boundary<C, ROWS>(a, p, cta + n) < tile_end) ++n;
  return n;
}

// ---- loading, by a warp
// A chunk of cached positions as TMA boxes, a lane each.  Page ids are read ahead of the wait for a place in the ring.
// (Requests of a warp go out one after the other, some 75 ns each: several warps share a chunk's, one map or half each.)
template <int C>
struct Ids {
  int id[C / 32], in_page;              // of the lane's box: id[0] and its first slot in the page; of rows that are copied: row 32 j + lane.  -1: none
};
template <int C>
__device__ inline void fetch_ids(const Args& a, const Seq& s, const Chunk& k, int lane, Ids<C>& x) {
  if (k.tree) return;
  const int* table = a.table + (int64_t)s.seq * a.max_pages;
  if (boxed(a, k)) {
    const int rows = a.box_rows, slot = place_of(a, k.start + lane * rows), pi = a.page_div(slot);      // (boxes of 4 slots and more, 2 of a chunk of 64: a lane each)
    x.id[0] = lane * rows < k.n ? table[pi] : -1;
    x.in_page = slot - pi * a.page_div.d;
  } else {
#pragma unroll
    for (int j = 0; j < C / 32; ++j) x.id[j] = 32 * j + lane < k.n ? table[a.page_div(place_of(a, k.start + 32 * j + lane))] : -1;
  }
}
// boxes first, first + step, ... of 64 features from `x0` to `to` (rows of 128 bytes); every lane arrives on the barrier once
template <int C>
__device__ inline void request_boxes(const Args& a, const CUtensorMap* map, int x0, const Chunk& k, const Ids<C>& x, int first, int step, int hk, unsigned char* to,
                                     uint64_t* bar, int lane) {
  const int rows = a.box_rows;
  const bool mine = lane * rows < k.n && lane % step == first, ok = mine && x.id[0] >= 0 && x.id[0] < a.n_pages;
  if (mine && !ok) {                                         // no page: zeros, and the caller is told
    if (a.status != nullptr) atomicMin(a.status, FM_ERR_INVALID_ARG);
    for (int i = 0; i < rows * 8; ++i) reinterpret_cast<uint4*>(to + lane * rows * 128)[i] = make_uint4(0u, 0u, 0u, 0u);
    ptx::fence_proxy_async();
  }
  const int n = __popc(__ballot_sync(0xffffffffu, ok));
  if (lane == 0) ptx::mbar_expect_tx(bar, (uint32_t)(n * rows * 128)); else ptx::mbar_arrive(bar);
  __syncwarp();
  if (ok) ptx::tma_load_4d(to + lane * rows * 128, map, x0, x.in_page, hk, x.id[0], bar);
  __syncwarp();
}
// The same with 16-byte copies, also for nodes; what is not there is zero.  By `threads` threads, the calling one is `t`;
// the copies are theirs (cp.async).  A warp's lanes share a group of 32 rows at a time.  KV: 0 keys, 1 values, 2 both.
template <typename T, int DH, int C, int KV>
__device__ inline void request_pieces(const Args& a, const Seq& s, const Chunk& k, int hk, unsigned char* Ks, unsigned char* Vs, const Ids<C>& x, int t, int threads) {
  constexpr int PIECES = DH / 8;
  const int piece = t % PIECES, step = threads / PIECES;
  const uint32_t ks = ptx::smem_u32(Ks) + (piece >> 3) * C * 128, vs = ptx::smem_u32(Vs) + (piece >> 3) * C * 128;
#pragma unroll 4
  for (int r = t / PIECES; r < C; r += step) {
    int group = x.id[0];
#pragma unroll
    for (int j = 1; j < C / 32; ++j) if (r >> 5 == j) group = x.id[j];
    const int id = __shfl_sync(0xffffffffu, group, r & 31);
    bool there = r < k.n;
    const T *kp = reinterpret_cast<const T*>(a.k), *vp = reinterpret_cast<const T*>(a.v);
    int64_t at = 0;
    if (k.tree) {
      kp = static_cast<const T*>(a.k_new); vp = static_cast<const T*>(a.v_new);
      if (there) at = (int64_t)(s.r0 + k.start + r) * a.new_row + hk * DH;
    } else if (there) {
      const int slot = place_of(a, k.start + r), pi = a.page_div(slot);
      if (id < 0 || id >= a.n_pages) {
        there = false;
        if (a.status != nullptr) atomicMin(a.status, FM_ERR_INVALID_ARG);
      } else {
        at = id * a.page + hk * a.head + (int64_t)(slot - pi * a.page_div.d) * a.slot;
      }
    }
    const uint32_t to = ptx::swz128(r, piece & 7);
    if (KV != 1) cp16(ks + to, kp + at + piece * 8, there);
    if (KV != 0) cp16(vs + to, vp + at + piece * 8, there);
  }
}
// query rows of a tile, behind the last one zeros; halves of ROWS x 128 bytes
template <typename T, int DH, int ROWS>
__device__ inline void request_queries(const Args& a, const Seq& s, int hk, int mt, unsigned char* Q, int t, int threads) {
  constexpr int PIECES = DH / 8;
  const int piece = t % PIECES, M = s.n * a.G, step = threads / PIECES;
  const uint32_t qs = ptx::smem_u32(Q) + (piece >> 3) * ROWS * 128;
#pragma unroll 4
  for (int r = t / PIECES; r < ROWS; r += step) {
    const int idx = mt * ROWS + r;
    const bool there = idx < M;
    const int node = there ? a.g_div(idx) : 0, gh = there ? idx - node * a.G : 0;
    cp16(qs + ptx::swz128(r, piece & 7), static_cast<const T*>(a.q) + (int64_t)(s.r0 + node) * a.q_row + (hk * a.G + gh) * DH + piece * 8, there);
  }
}
// after the last request: who else has parts of the tile that this CTA starts and does not end
template <int C, int ROWS>
__device__ inline void write_desc(const Args& a, const Plan& p, int4 cut, long long cut_end, int lane) {
  if (lane == 0) {
    if (cut.w != 0) cut.w = parts_of<C, ROWS>(a, p, blockIdx.x, cut_end);
    a.desc[blockIdx.x] = cut;
  }
}

// ---- ancestors of the nodes of a sequence, by `threads` threads that meet at `bar`: reach[i] (zero: not in use), depth[i]
struct Tree {
  uint32_t reach[FM_MAX_TREE_NODES][WORDS];
  short jump[FM_MAX_TREE_NODES];
  short depth[FM_MAX_TREE_NODES];
  int max_depth;
};
// Which of the keys k0 .. k0 + 31 of a chunk a row sees, a bit each (k0 a multiple of 16, a tree's chunks start at multiples of
// 32; of a k0 that is none of 32 the lower 16 bits count).  node: the row's, -1: none; low: the first cached position it sees.
__device__ inline uint32_t seen(const Args& a, const Tree& t, const Chunk& ck, int node, int depth, int low, int k0) {
  auto below = [](int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); };
  const int at = ck.start + k0;
  if (node < 0 || k0 >= ck.n) return 0u;
  if (!ck.tree) return (below(a.n_prefix - at) | ~below(low - at)) & below(ck.n - k0);
  uint32_t bits = t.reach[node][at >> 5] >> (at & 31);
  if (a.window > 0 && depth >= a.window)
    for (uint32_t left = bits; left != 0u; left &= left - 1u)
      if (depth - t.depth[at + __ffs(left) - 1] >= a.window) bits &= ~(left & (0u - left));
  return bits;
}
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
// Eight warps multiply: four take the even chunks, four the odd ones, each a fixed slice of a chunk with its own running maximum,
// sum and output (base 2).  At the end of a tile one of the two groups hands its states over and goes on, the other merges
// and writes: they take turns.  Four warps load, queries and parents of the next tile included.
// Bound: memory, once the SMs are full: 64 sequences of 4000 positions, 8 kv-heads of 128, one node: 176 us, 5.96 TB/s (91 % of a
// copy); the same of 100 to 8000 positions in pages of 16: 102 us, 4.6 TB/s (70 %: pieces of 4 KB, parts and merges of ragged shares).
// A pass of four nodes over 150 positions takes 8.6 us: a launch, the plan, a chunk's latency and the end of a tile.
template <int DH>
struct Rows16 {
  static constexpr int ROWS = 16, C = DH == 64 ? 128 : 64, NW = 4, KPW = C / NW, STAGES = 4;
  static constexpr int TILE = C * DH * 2, STAGE = 2 * TILE, RING = STAGES * STAGE, Q = 16 * DH * 2;
  static constexpr int STATES = NW * 16 * (DH + 2) * 4;
  static constexpr int THREADS = 2 * NW * 32 + 128;
  static constexpr int PARENTS = FM_MAX_TREE_NODES * 4;
  static constexpr int FIXED = RING + 2 * Q + 2 * PARENTS + STATES + (int)sizeof(Tree) + 1024 + 512;
  static int bytes(int batch) { return FIXED + plan_bytes(batch); }
};

template <typename T, int DH>
__global__ void __launch_bounds__(Rows16<DH>::THREADS, 1) rows16_kernel(const __grid_constant__ Args a) {
  using CF = Rows16<DH>;
  constexpr int C = CF::C, NW = CF::NW, KPW = CF::KPW, KS = DH / 16, KB = KPW / 16, NT = KPW / 8, ST = CF::STAGES;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* sq = sm + CF::RING;                         // [2] queries
  int* s_parent = reinterpret_cast<int*>(sq + 2 * CF::Q);    // [2] parents of the tile's sequence
  float* pw = reinterpret_cast<float*>(s_parent + 2 * FM_MAX_TREE_NODES);      // [NW][16][DH] outputs
  float* ml = pw + NW * 16 * DH;                             // [NW][16][2] maxima and sums
  int4* s_info = reinterpret_cast<int4*>(pw + NW * 16 * (DH + 2));
  long long* s_base = reinterpret_cast<long long*>(s_info + a.batch);
  long long* s_sh = s_base + a.batch + 1;                    // [2 * warps]
  uint64_t* full = reinterpret_cast<uint64_t*>(s_sh + 24);
  uint64_t *empty = full + ST, *q_full = empty + ST, *q_free = q_full + 2;
  Tree& tree = *reinterpret_cast<Tree*>(q_free + 2);
  int* s_tile_base = reinterpret_cast<int*>(&tree + 1);
  __shared__ int s_fail;
  const int warp = (int)ptx::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  if (threadIdx.x == 0) {
    s_fail = 0;
    for (int i = 0; i < ST; ++i) { ptx::mbar_init(full + i, 128); ptx::mbar_init(empty + i, NW); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(q_full + i, 128); ptx::mbar_init(q_free + i, 2 * NW); }
    ptx::fence_mbar_init();
  }
  Plan plan;
  const int2 ends = ends_of(a);
  make_plan<C, 16, CF::THREADS>(a, plan, s_info, s_base, s_tile_base, s_sh);
  if (to_fill(a, plan, ends)) fill<DH>(a, plan, ends);
  Walk<C, 16> w;
  w.init(a, plan, blockIdx.x);
  auto wait = [](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity)) != 0; };
  __syncthreads();

  if (warp >= 2 * NW) {
    // ---- loading: warps 0 and 2 keys, 1 and 3 values; of 128 features half each, of 64 every other box
    const int lw = warp - 2 * NW, tid = threadIdx.x - 2 * NW * 32;
    const CUtensorMap* map = (lw & 1) ? &a.map_v : &a.map_k;
    const int x0 = DH == 128 ? (lw >> 1) * 64 : 0, first = DH == 128 ? 0 : lw >> 1, step = DH == 128 ? 1 : 2;
    const int off = (lw & 1) * CF::TILE + (DH == 128 ? (lw >> 1) * C * 128 : 0);
    int i = 0, part = 0, written = 0;                        // chunks left whose place threads have written
    int4 cut = make_int4(0, 0, 0, 0);
    long long cut_end = 0;
    bool ok = true;
    while (ok && w.next(a, plan)) {
      const int hk = w.hk, mt = w.mt;
      if (w.starts() && !w.ends()) { cut = make_int4(w.b, hk, mt, 1); cut_end = w.tile_start + w.s.chunks + OVER; }
      if (part >= 2 && !(ok = wait(q_free + (part & 1), ((part >> 1) - 1) & 1))) break;
      request_queries<T, DH, 16>(a, w.s, hk, mt, sq + (part & 1) * CF::Q, tid, 128);
      for (int j = tid; j < w.s.n; j += 128)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(ptx::smem_u32(s_parent + (part & 1) * FM_MAX_TREE_NODES + j)), "l"(a.parent + w.s.r0 + j) : "memory");
      cp_arrive(q_full + (part & 1));
      ++part;
      Chunk k = chunk_of<C>(w.s, w.c);
      Ids<C> x;
      fetch_ids<C>(a, w.s, k, lane, x);
      for (int c = w.c; c < w.c_end; ++c, ++i) {
        const int st = i % ST;
        if (i >= ST && !(ok = wait(empty + st, ((i / ST) - 1) & 1))) break;
        unsigned char* Ks = sm + st * CF::STAGE;
        if (boxed(a, k)) {
          if (written > 0) { --written; ptx::fence_proxy_async(); }
          request_boxes<C>(a, map, x0, k, x, first, step, hk, Ks + off, full + st, lane);
        } else {
          request_pieces<T, DH, C, 2>(a, w.s, k, hk, Ks, Ks + CF::TILE, x, tid, 128);
          cp_arrive(full + st);
          written = ST;
        }
        if (c + 1 < w.c_end) { k = chunk_of<C>(w.s, c + 1); fetch_ids<C>(a, w.s, k, lane, x); }
      }
    }
    if (!ok) s_fail = 1;
    if (lw == 0) write_desc<C, 16>(a, plan, cut, cut_end, lane);
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    // ---- multiplying
    auto sync = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    const int group = warp >> 2, wg = warp & 3;
    int tree_of = -1, it = 0, part = 0;
    bool ok = true;                                          // (when a wait has given up the warps still meet at their barriers)
    while (w.next(a, plan)) {
      const Seq& s = w.s;
      const int hk = w.hk, mt = w.mt, M = s.n * a.G;
      const bool whole = w.starts() && w.ends();
      ok = ok && wait(q_full + (part & 1), (part >> 1) & 1);
      if (tree_of != w.b) { build_tree<256>(tree, s_parent + (part & 1) * FM_MAX_TREE_NODES, s.n, threadIdx.x, sync); tree_of = w.b; }
      uint32_t qa[KS][4];
      {
        const uint32_t q = ptx::smem_u32(sq + (part & 1) * CF::Q);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int ch = ks * 2 + (lane >> 4);
          ptx::ldmatrix_x4(qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], q + (ch >> 3) * 16 * 128 + ptx::swz128(lane & 15, ch & 7));
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(q_free + (part & 1));
      }
      // the rows' nodes (-1: behind the last), depths, first cached positions behind the prefix that they see
      int node[2], depth[2], low[2];
#pragma unroll
      for (int hr = 0; hr < 2; ++hr) {
        const int idx = mt * 16 + g + hr * 8;
        node[hr] = idx < M ? a.g_div(idx) : -1;
        depth[hr] = node[hr] >= 0 ? tree.depth[node[hr]] : 0;
        low[hr] = a.window > 0 ? s.len + depth[hr] - a.window + 1 : 0;
      }
      const int low_all = a.window > 0 ? s.len + tree.max_depth - a.window + 1 : 0;
      float o[DH / 8][4];
      float mrun[2] = {-INFINITY, -INFINITY}, lrun[2] = {0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DH / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
      for (int c = w.c; c < w.c_end; ++c, ++it) {
        if ((it & 1) != group) continue;
        const Chunk ck = chunk_of<C>(s, c);
        const int st = it % ST;
        const bool uneven = ck.tree || (a.window > 0 && ck.start + ck.n > a.n_prefix && ck.start < low_all);   // rows differ in what they see
        const bool all_vis = !uneven && ck.n == C;
        if (!(ok = ok && wait(full + st, (it / ST) & 1))) break;
        const uint32_t Ks_u = ptx::smem_u32(sm + st * CF::STAGE), Vs_u = Ks_u + CF::TILE;
        uint32_t kf[KB][KS][4], vf[KB][DH / 16][4];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const int key = wg * KPW + kb * 16 + (lane & 7) + (lane >> 4) * 8;
            const int ch = ks * 2 + ((lane >> 3) & 1);
            ptx::ldmatrix_x4(kf[kb][ks][0], kf[kb][ks][1], kf[kb][ks][2], kf[kb][ks][3], Ks_u + (ch >> 3) * C * 128 + ptx::swz128(key, ch & 7));
          }
        // (128 features: behind the scores, or keys and values together take more registers than there are)
        auto load_values = [&] {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int dp = 0; dp < DH / 16; ++dp) {
              const int key = wg * KPW + kb * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
              const int ch = dp * 2 + (lane >> 4);
              ptx::ldmatrix_x4_trans(vf[kb][dp][0], vf[kb][dp][1], vf[kb][dp][2], vf[kb][dp][3], Vs_u + (ch >> 3) * C * 128 + ptx::swz128(key, ch & 7));
            }
        };
        if (DH == 64) load_values();
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
        if (DH == 128) load_values();
        bool bad = false;
        if (!all_vis) {
          // keys of this thread: n-tile nt, element e -> nt * 8 + 2 * t4 + e of the warp's slice
#pragma unroll
          for (int hr = 0; hr < 2; ++hr) {
            const uint32_t bits = seen(a, tree, ck, node[hr], depth[hr], low[hr], wg * KPW) >> (2 * t4);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (!((bits >> (nt * 8 + e)) & 1u)) sc[nt][hr * 2 + e] = -INFINITY;
          }
          // (what lies behind the length is whatever the page holds)
          uint32_t most = 0u;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int dp = 0; dp < DH / 16; ++dp)
#pragma unroll
              for (int j = 0; j < 4; ++j) most = largest<T>(most, vf[kb][dp][j]);
          (void)finite_part<T>(most, bad);
          if (bad) {
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
          const float mnew = fmaxf(mrun[hr], fmaf(mx, a.scale_log2, -SHIFT<T>));
          base[hr] = mnew == -INFINITY ? 0.f : mnew;
          scale[hr] = mnew == mrun[hr] ? 1.f : ex2(mrun[hr] - base[hr]);
          mrun[hr] = mnew;
        }
        float ls[2] = {0.f, 0.f};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sc[nt][e] = ex2(fmaf(sc[nt][e], a.scale_log2, -base[e >> 1]));
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
              const int key = wg * KPW + nt * 8 + k, src = (lane & ~3) | (k >> 1);
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
      if (!ok) s_fail = 1;
#pragma unroll
      for (int hr = 0; hr < 2; ++hr) {
        lrun[hr] += __shfl_xor_sync(0xffffffffu, lrun[hr], 1);
        lrun[hr] += __shfl_xor_sync(0xffffffffu, lrun[hr], 2);
      }
      // ---- the states: one group's to the same warps of the other, then those in warp order.  The groups take turns, so the
      // one that writes states is the one that read the last ones.  Barriers 2 and 3 (the states are there) take turns too: a
      // group may be a tile ahead of the other, not two.
      float* mine = pw + wg * 16 * DH;
      auto put = [&] {
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) {
          *reinterpret_cast<float2*>(mine + g * DH + i * 8 + 2 * t4) = make_float2(o[i][0], o[i][1]);
          *reinterpret_cast<float2*>(mine + (g + 8) * DH + i * 8 + 2 * t4) = make_float2(o[i][2], o[i][3]);
        }
        if (t4 == 0) {
          *reinterpret_cast<float2*>(ml + (wg * 16 + g) * 2) = make_float2(mrun[0], lrun[0]);
          *reinterpret_cast<float2*>(ml + (wg * 16 + g + 8) * 2) = make_float2(mrun[1], lrun[1]);
        }
      };
      const int odd = part++ & 1;
      if (group != odd) {
        put();
        asm volatile("bar.arrive %0, 256;" ::"r"(2 + odd) : "memory");
        continue;
      }
      asm volatile("bar.sync %0, 256;" ::"r"(2 + odd) : "memory");
#pragma unroll
      for (int hr = 0; hr < 2; ++hr) {
        const float2 q = *reinterpret_cast<const float2*>(ml + (wg * 16 + g + 8 * hr) * 2);
        // (no chunk on one side: maximum -inf and sum 0; a sum that is no number goes through)
        const float mm = fmaxf(mrun[hr], q.x), f0 = mrun[hr] == -INFINITY ? 1.f : ex2(mrun[hr] - mm), f1 = q.x == -INFINITY ? 1.f : ex2(q.x - mm);
        lrun[hr] = (f0 == 0.f ? 0.f : lrun[hr] * f0) + (f1 == 0.f ? 0.f : q.y * f1);
        mrun[hr] = mm;
#pragma unroll
        for (int i = 0; i < DH / 8; ++i) {
          const float2 v = *reinterpret_cast<const float2*>(mine + (g + 8 * hr) * DH + i * 8 + 2 * t4);
          o[i][2 * hr] = (f0 == 0.f ? 0.f : o[i][2 * hr] * f0) + (f1 == 0.f ? 0.f : v.x * f1);
          o[i][2 * hr + 1] = (f0 == 0.f ? 0.f : o[i][2 * hr + 1] * f0) + (f1 == 0.f ? 0.f : v.y * f1);
        }
      }
      __syncwarp();
      put();
      auto sync4 = [&] { asm volatile("bar.sync %0, 128;" ::"r"(4 + group) : "memory"); };
      sync4();
      const int rows_here = min(16, M - mt * 16);
      float* part_at = a.part + (size_t)(blockIdx.x * 2 + (w.starts() ? 1 : 0)) * 16 * (DH + 2);
      for (int e = threadIdx.x & 127; e < rows_here * (DH / 2); e += 128) {
        const int i = e / (DH / 2), col = 2 * (e - i * (DH / 2)), idx = mt * 16 + i, nd = a.g_div(idx), gh = idx - nd * a.G;
        const bool live = tree.reach[nd][nd >> 5] != 0u;
        float2 stt[NW];
        float mm = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) { stt[k] = *reinterpret_cast<const float2*>(ml + (k * 16 + i) * 2); mm = fmaxf(mm, stt[k].x); }
#pragma unroll
        for (int k = 0; k < NW; ++k) {
          const float f = stt[k].x == -INFINITY ? 1.f : ex2(stt[k].x - mm);
          const float2 v = *reinterpret_cast<const float2*>(pw + (k * 16 + i) * DH + col);
          if (f != 0.f) { l += f * stt[k].y; o0 += f * v.x; o1 += f * v.y; }
        }
        if (!live) { mm = -INFINITY; l = o0 = o1 = 0.f; }
        if (whole) {
          const float inv = live ? 1.f / l : 0.f;
          T* at = static_cast<T*>(a.out) + (int64_t)(s.r0 + nd) * a.out_row + (hk * a.G + gh) * DH + col;
          const uint32_t hi = pack(o0 * inv, o1 * inv, T());
          *reinterpret_cast<uint32_t*>(at) = hi;
          if (a.lo_off > 0) *reinterpret_cast<uint32_t*>(at + a.lo_off) = pack_rest(o0 * inv, o1 * inv, hi);
          if (col == 0 && a.lse != nullptr) a.lse[(int64_t)(s.r0 + nd) * a.H + hk * a.G + gh] = live ? (mm + log2f(l)) * 0.6931471805599453f : -INFINITY;
        } else {
          float* row = part_at + (size_t)i * (DH + 2);
          *reinterpret_cast<float2*>(row + col) = make_float2(o0, o1);
          if (col == 0) *reinterpret_cast<float2*>(row + DH) = make_float2(mm, l);
        }
      }
      sync4();                                               // the states have been read
    }
  }
  __syncthreads();
  if (s_fail) {                                              // a bounded wait gave up: report, once what was requested has landed
    if (threadIdx.x == 0 && a.status != nullptr) atomicMin(a.status, FM_ERR_TIMEOUT);
    ptx::drain_delay();
  }
}

// ------------------------------------------------------------------------------------------
// 256 query rows a tile, on the tensor cores
// ------------------------------------------------------------------------------------------
// S = Q K^T and O += P V are tcgen05 MMAs with accumulators in tensor memory; V is multiplied as it lies (keys x features:
// MN-major), P goes back to tensor memory as the A operand.  Two slots work in turn, each with its S, P and O and four warps
// of softmax, a thread a row: one's exponentials run under the other's products.  A tile of more than 128 rows gives each slot
// half of them and every chunk to both (keys and values are loaded once for 256 rows); one of up to 128 rows gives its
// chunks to the slots alternately, and their outputs are merged at the end.  Steps are numbered through: slot = step mod 2.
// Exponentials are taken to the maximum in use, that of the row's first chunk, and the scores' maximum beside them: only when it
// exceeds the one in use by more than P's type holds (2^40 for bfloat16, 2^6.5 for half, whose weights start at 2^9: see SHIFT) the output
// is rescaled and the chunk's exponentials are taken again.  (The maximum first, then the exponentials: a step of a slot took 4200 clocks, 560
// of them for the maximum.)
// One warp brings keys, one values, each as soon as its place is free (keys once their scores are multiplied); a third
// one (the fixer) brings queries and takes values that are not finite out of chunks with hidden keys.  What threads write is
// made visible to the tensor cores by a proxy fence.
// Bound: the special-function units (1024 clocks for the exponentials of 128 rows x 128 keys, about what the products of
// heads of 128 take) and, between them and the products, the latency of a slot's turn: 1800 clocks a step of 128 x 128.  Eight
// sequences of 32768 positions, 64 nodes: 8 kv-heads of 128, 4 heads a group 318 us (866 TFLOP/s, at the power limit); 4
// kv-heads of 64, 8 heads a group 262 us (525).  Few rows: 28 nodes, 16 sequences of 9000, 16 heads of 64: 174 us, 3.4 TB/s.
template <int DH>
struct Rows256 {
  static constexpr int ROWS = 256, C = 128, STAGES = DH == 64 ? 4 : 2;
  static constexpr int THREADS = 128 + 256;                  // keys, fixer, MMA, values; softmax
  static constexpr int Q = 128 * DH * 2, TILE = C * DH * 2, STAGE = 2 * TILE;
  // tensor memory, columns: S of both slots, O of both; P of heads of 64 behind them, of heads of 128 in the place of S
  static constexpr bool ALIAS = DH == 128;
  static constexpr int O_AT = 2 * C, P_AT = O_AT + 2 * DH;
  static_assert(P_AT + (ALIAS ? 0 : 2 * C / 2) <= 512, "");
  static constexpr int FIXED = 2 * Q + STAGES * STAGE + (int)sizeof(Tree) + 2 * 128 * 8 + 512 + 1024;
  static int bytes(int batch) { return FIXED + plan_bytes(batch); }
};
// log2 of what P may grow to, and of what it starts at: of half's 40 powers of two 6.5 for growth, 34 below the first chunk's maximum
template <typename T> constexpr float HEADROOM = __is_same(T, bf16) ? 40.f : 15.5f;
template <typename T> constexpr float START = __is_same(T, bf16) ? 0.f : 9.f;

__device__ inline uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ inline float2 unpack2(uint64_t r) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
  return v;
}
__device__ inline uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ inline uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ inline float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ inline void st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
               : "memory");
}
__device__ inline void ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,"
      "%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr));
}
__device__ inline void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ inline void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ inline void mma_ts(uint32_t d, uint32_t a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
// fp32 accumulate, A and B of type T, M = 128, N = n
template <typename T>
__device__ constexpr uint32_t instr_desc(int n) {
  return (1u << 4) | (__is_same(T, bf16) ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// Can a chunk hold keys that some row does not see?  (The deepest node has fewer ancestors than the tree has nodes.  What lies
// behind the length is whatever the page holds.)
template <int C>
__device__ inline bool uneven_chunk(const Args& a, const Seq& s, const Chunk& k) {
  return k.tree || k.n < C || (a.window > 0 && k.start + k.n > a.n_prefix && k.start < s.len + s.n - a.window);
}
// values of a key: where they are, null if its page is none
template <typename T, int DH>
__device__ inline const T* values_of(const Args& a, const Seq& s, const Chunk& k, int hk, int key) {
  if (k.tree) return static_cast<const T*>(a.v_new) + (int64_t)(s.r0 + k.start + key) * a.new_row + hk * DH;
  const int at = place_of(a, k.start + key), pi = a.page_div(at), id = a.table[(int64_t)s.seq * a.max_pages + pi];
  if (id < 0 || id >= a.n_pages) return nullptr;
  return reinterpret_cast<const T*>(a.v) + id * a.page + hk * a.head + (int64_t)(at - pi * a.page_div.d) * a.slot;
}

template <typename T, int DH>
__global__ void __launch_bounds__(Rows256<DH>::THREADS, 1) rows256_kernel(const __grid_constant__ Args a) {
  using CF = Rows256<DH>;
  constexpr int C = CF::C, ST = CF::STAGES, TILE = CF::TILE, STAGE = CF::STAGE;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* ring = sm + 2 * CF::Q;                      // behind the queries
  float2* s_ml = reinterpret_cast<float2*>(ring + ST * STAGE);             // [slot][row] maxima and sums
  int4* s_info = reinterpret_cast<int4*>(s_ml + 256);
  long long* s_base = reinterpret_cast<long long*>(s_info + a.batch);
  long long* s_sh = s_base + a.batch + 1;                    // [2 * warps]
  uint64_t* full = reinterpret_cast<uint64_t*>(s_sh + 24);
  uint64_t *full_v = full + ST, *fixed = full_v + ST, *free_k = fixed + ST, *free_v = free_k + ST, *q_full = free_v + ST, *q_free = q_full + 1,
           *s_full = q_free + 1, *p_full = s_full + 2, *o_full = p_full + 2, *done = o_full + 2;           // (the last four: a slot each)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  Tree& tree = *reinterpret_cast<Tree*>(done + 2);
  int* s_tile_base = reinterpret_cast<int*>(&tree + 1);
  __shared__ int s_fail, s_bad;
  const int warp = (int)ptx::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  ptx::grid_dep_wait();
  if (threadIdx.x == 0) {
    s_fail = s_bad = 0;
    for (int i = 0; i < ST; ++i) {
      ptx::mbar_init(full + i, 32); ptx::mbar_init(full_v + i, 32); ptx::mbar_init(fixed + i, 32);
      ptx::mbar_init(free_k + i, 1); ptx::mbar_init(free_v + i, 1);
    }
    ptx::mbar_init(q_full, 32); ptx::mbar_init(q_free, 1); ptx::mbar_init(done, 1);
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(s_full + i, 1); ptx::mbar_init(p_full + i, 4); ptx::mbar_init(o_full + i, 1); }
    ptx::fence_mbar_init();
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  Plan plan;
  const int2 ends = ends_of(a);
  make_plan<C, 256, CF::THREADS>(a, plan, s_info, s_base, s_tile_base, s_sh);
  if (to_fill(a, plan, ends)) fill<DH>(a, plan, ends);
  Walk<C, 256> w;
  w.init(a, plan, blockIdx.x);
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = ptx::uniform(*tmem_slot);
  ptx::grid_dep_launch();                                    // (not before: a dependent's block on this SM may hold tensor memory while it waits for this grid)
  auto wait = [](uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity)) != 0; };
  auto two = [&] { return w.s.n * a.G - w.mt * 256 > 128; };               // more than 128 rows in the tile

  if (warp == 0 || warp == 3) {
    // ---- keys, values
    const bool v = warp == 3;
    uint64_t *mine = v ? full_v : full, *room = v ? free_v : free_k;
    int i = 0;
    int4 cut = make_int4(0, 0, 0, 0);
    long long cut_end = 0;
    bool ok = true;
    while (ok && w.next(a, plan)) {
      const int hk = w.hk;
      if (w.starts() && !w.ends()) { cut = make_int4(w.b, hk, w.mt, 1); cut_end = w.tile_start + w.s.chunks + OVER; }
      Chunk k = chunk_of<C>(w.s, w.c);
      Ids<C> x;
      fetch_ids<C>(a, w.s, k, lane, x);
      for (int c = w.c; c < w.c_end; ++c, ++i) {
        const int st = i % ST;
        unsigned char *Ks = ring + st * STAGE, *Vs = Ks + TILE;
        if (i >= ST && !(ok = wait(room + st, ((i / ST) - 1) & 1))) break;
        if (boxed(a, k)) {
          // (both halves of a box in a lane: they land on one barrier, which every lane arrives on once)
          const CUtensorMap* map = v ? &a.map_v : &a.map_k;
          const int rows = a.box_rows;
          const bool has = lane * rows < k.n, good = has && x.id[0] >= 0 && x.id[0] < a.n_pages;
          unsigned char* to = (v ? Vs : Ks) + lane * rows * 128;
          if (has && !good) {                                // no page: zeros, and the caller is told
            if (a.status != nullptr) atomicMin(a.status, FM_ERR_INVALID_ARG);
            for (int h = 0; h < DH / 64; ++h)
              for (int j = 0; j < rows * 8; ++j) reinterpret_cast<uint4*>(to + h * C * 128)[j] = make_uint4(0u, 0u, 0u, 0u);
            ptx::fence_proxy_async();
          }
          const int n = __popc(__ballot_sync(0xffffffffu, good));
          if (lane == 0) ptx::mbar_expect_tx(mine + st, (uint32_t)(n * rows * 128 * (DH / 64))); else ptx::mbar_arrive(mine + st);
          __syncwarp();
          if (good) {
#pragma unroll
            for (int h = 0; h < DH / 64; ++h) ptx::tma_load_4d(to + h * C * 128, map, h * 64, x.in_page, hk, x.id[0], mine + st);
          }
          __syncwarp();
        } else {
          if (v) request_pieces<T, DH, C, 1>(a, w.s, k, hk, Ks, Vs, x, lane, 32); else request_pieces<T, DH, C, 0>(a, w.s, k, hk, Ks, Vs, x, lane, 32);
          asm volatile("cp.async.wait_all;" ::: "memory");
          ptx::fence_proxy_async();
          ptx::mbar_arrive(mine + st);
        }
        if (c + 1 < w.c_end) { k = chunk_of<C>(w.s, c + 1); fetch_ids<C>(a, w.s, k, lane, x); }
      }
    }
    if (!ok) s_fail = 1;
    if (!v) write_desc<C, 256>(a, plan, cut, cut_end, lane);
  } else if (warp == 1) {
    // ---- fixing
    int i = 0, part = 0;
    bool ok = true;
    while (ok && w.next(a, plan)) {
      // the tile's queries, once the scores of the tile before have been multiplied
      if (part > 0 && !(ok = wait(q_free, (part - 1) & 1))) break;
      request_queries<T, DH, 128>(a, w.s, w.hk, 2 * w.mt, sm, lane, 32);
      if (two()) request_queries<T, DH, 128>(a, w.s, w.hk, 2 * w.mt + 1, sm + CF::Q, lane, 32);
      asm volatile("cp.async.wait_all;" ::: "memory");
      ptx::fence_proxy_async();
      ptx::mbar_arrive(q_full);
      ++part;
      for (int c = w.c; c < w.c_end; ++c, ++i) {
        const Chunk k = chunk_of<C>(w.s, c);
        const int st = i % ST;
        // (for every chunk: this warp must not fall two phases behind a barrier, a parity tells two apart, nor run ahead)
        if (!(ok = wait(full_v + st, (i / ST) & 1))) break;
        if (uneven_chunk<C>(a, w.s, k)) {
          uint4* Vs = reinterpret_cast<uint4*>(ring + st * STAGE + TILE);
          bool bad = false;
          for (int j = lane; j < TILE / 16; j += 32) {
            uint4 u = Vs[j];
            bool here = false;
            u.x = finite_part<T>(u.x, here); u.y = finite_part<T>(u.y, here); u.z = finite_part<T>(u.z, here); u.w = finite_part<T>(u.w, here);
            if (here) { Vs[j] = u; bad = true; }
          }
          if (bad) *reinterpret_cast<volatile int*>(&s_bad) = 1;
          ptx::fence_proxy_async();
        }
        ptx::mbar_arrive(fixed + st);
      }
    }
    if (!ok) s_fail = 1;
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == 2) {
    // ---- multiplying.  Scores run two steps ahead of the products with values, inside a tile.
    const uint32_t id_s = instr_desc<T>(C), id_o = instr_desc<T>(DH) | (1u << 16);          // B of P V is MN-major
    const uint64_t dq = tc::smem_desc_sw128(ptx::smem_u32(sm));
    int g = 0, it = 0, part = 0;                             // step, chunk of the ring, tile
    bool ok = true;
    while (ok && w.next(a, plan)) {
      const int per = two() ? 2 : 1, steps = (w.c_end - w.c) * per;        // steps a chunk, steps of the tile
      if (!(ok = wait(q_full, part++ & 1))) break;
      auto scores = [&](int k) {                             // step k of the tile
        const int i = it + k / per, st = i % ST, slot = (g + k) & 1, sub = per == 2 ? k & 1 : 0;
        const bool first_of = per == 1 || sub == 0, last_of = per == 1 || sub == 1;
        if (first_of && !wait(full + st, (i / ST) & 1)) return false;
        // the slot's last product has read P where the scores go (heads of 128), its last softmax the scores
        if (CF::ALIAS && g + k >= 2 && !wait(o_full + slot, ((g + k - 2) >> 1) & 1)) return false;
        tc::fence_after();
        const uint64_t q = dq + sub * (CF::Q / 16), dk = tc::smem_desc_sw128(ptx::smem_u32(ring + st * STAGE));
        if (ptx::elect_one()) {
#pragma unroll
          for (int j = 0; j < DH / 16; ++j)                  // 64 features a half, 16 a step
            tc::mma_ss(tmem + slot * C, q + (j >> 2) * (128 * 128 / 16) + 2 * (j & 3), dk + (j >> 2) * (C * 128 / 16) + 2 * (j & 3), id_s, j > 0 ? 1u : 0u);
          tc::commit(s_full + slot);                         // (counts when all that was issued before is done: the slot's last product too)
          if (last_of) tc::commit(free_k + st);
          if (k == steps - 1) tc::commit(q_free);
        }
        return true;
      };
      ok = scores(0) && (steps < 2 || scores(1));
      for (int k = 0; k < steps && ok; ++k) {
        const int i = it + k / per, st = i % ST, slot = (g + k) & 1, sub = per == 2 ? k & 1 : 0;
        if (sub == 0 && !(ok = wait(full_v + st, (i / ST) & 1) && wait(fixed + st, (i / ST) & 1))) break;
        if (!(ok = wait(p_full + slot, ((g + k) >> 1) & 1))) break;
        tc::fence_after();
        // (MN-major: the leading offset is that between the halves of 64 features, the stride offset that between 8 keys)
        const uint64_t dv = tc::smem_desc_sw128(ptx::smem_u32(ring + st * STAGE + TILE)) + ((uint64_t)(C * 128 / 16 - 1) << 16);
        const uint32_t tO = tmem + CF::O_AT + slot * DH, tP = tmem + (CF::ALIAS ? slot * C : CF::P_AT + slot * C / 2);
        const bool fresh = k < 2;                            // the slot's first product of the tile
        if (ptx::elect_one()) {
#pragma unroll
          for (int j = 0; j < C / 16; ++j) mma_ts(tO, tP + 8 * j, dv + 128 * j, id_o, (!fresh || j > 0) ? 1u : 0u);
          tc::commit(o_full + slot);
          if (per == 1 || sub == 1) tc::commit(free_v + st);
        }
        if (k + 2 < steps) ok = scores(k + 2);
      }
      g += steps;
      it += w.c_end - w.c;
    }
    if (!ok) s_fail = 1;
    if (ptx::elect_one()) tc::commit(done);                  // what was issued ends before the CTA does
    wait(done, 0);
  } else {
    // ---- softmax: a slot's four warps, a thread a row
    const int w4 = warp & 3, slot = (warp - 4) >> 2, i_row = w4 * 32 + lane, tid = threadIdx.x - 128;
    const uint32_t lanes = (uint32_t)(w4 * 32) << 16, tS = tmem + slot * C + lanes, tO = tmem + CF::O_AT + slot * DH + lanes,
                   tP = CF::ALIAS ? tS : tmem + CF::P_AT + slot * C / 2 + lanes;
    auto sync = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
    const float sc = a.scale_log2;
    int tree_of = -1, g = 0;
    bool ok = true;
    while (w.next(a, plan)) {
      const Seq& s = w.s;
      const bool both = two();                               // two tiles of rows, or two shares of the chunks
      const int per = both ? 2 : 1, steps = (w.c_end - w.c) * per, k_first = (g + slot) & 1;               // the slot's first step of the tile: 0 or 1
      const int hk = w.hk, idx = w.mt * 256 + (both ? k_first * 128 : 0) + i_row, M = s.n * a.G;
      if (tree_of != w.b) { build_tree<256>(tree, a.parent + s.r0, s.n, tid, sync); tree_of = w.b; }
      const bool whole = w.starts() && w.ends(), there = idx < M;
      const int node = there ? a.g_div(idx) : 0, gh = there ? idx - node * a.G : 0, depth = there ? tree.depth[node] : 0;
      const int low = a.window > 0 ? s.len + depth - a.window + 1 : 0, low_all = a.window > 0 ? s.len + tree.max_depth - a.window + 1 : 0;
      float m = -INFINITY, l = 0.f;                          // the maximum in use (times scale, base 2), the sum
      bool any = false;
      for (int k = k_first; k < steps; k += 2) {
        const Chunk ck = chunk_of<C>(s, w.c + k / per);
        const int n = (g + k) >> 1;                          // the slot's step
        const bool all_vis = !ck.tree && ck.n == C && !(a.window > 0 && ck.start + C > a.n_prefix && ck.start < low_all);
        ok = ok && wait(s_full + slot, n & 1);               // (goes on: the warps meet at barriers)
        tc::fence_after();
        uint32_t bits[C / 32];
        if (!all_vis) {
#pragma unroll
          for (int q = 0; q < C / 32; ++q) bits[q] = seen(a, tree, ck, there ? node : -1, depth, low, 32 * q);
        }
        uint32_t r[2][32], pk[CF::ALIAS ? C / 32 : 1][16];
        auto block = [&](int q) -> uint32_t* {               // columns 32 q .. of the scores; the next ones are requested
          ld_wait();
          if (q + 1 < C / 32) ld32(tS + 32 * (q + 1), r[(q + 1) & 1]);
          uint32_t* x = r[q & 1];
          if (!all_vis) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!((bits[q] >> j) & 1u)) x[j] = 0xff800000u;              // -inf: exponential 0
          }
          return x;
        };
        float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        auto largest4 = [&](const uint32_t* x) {
#pragma unroll
          for (int j = 0; j < 32; j += 8)
#pragma unroll
            for (int u = 0; u < 4; ++u) m4[u] = max3(m4[u], __uint_as_float(x[j + 2 * u]), __uint_as_float(x[j + 2 * u + 1]));
        };
        auto row_max = [&] { return fmaf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), sc, -START<T>); };
        if (!any) {                                          // the row's first chunk: its maximum first
          ld32(tS, r[0]);
#pragma unroll
          for (int q = 0; q < C / 32; ++q) largest4(block(q));
          m = row_max();
        }
        float sum;
        while (true) {
          const float base = m == -INFINITY ? 0.f : m;
          const uint64_t nb = pack2(-base, -base), s2 = pack2(sc, sc);
          uint64_t sums[2] = {0ull, 0ull};
          ld32(tS, r[0]);
#pragma unroll
          for (int q = 0; q < C / 32; ++q) {
            const uint32_t* x = block(q);
            largest4(x);
            uint32_t(&p)[16] = pk[CF::ALIAS ? q : 0];
#pragma unroll
            for (int u = 0; u < 16; ++u) {
              const float2 d = unpack2(fma2(pack2(__uint_as_float(x[2 * u]), __uint_as_float(x[2 * u + 1])), s2, nb));
              const float e0 = ex2(d.x), e1 = ex2(d.y);
              sums[u & 1] = add2(sums[u & 1], pack2(e0, e1));
              p[u] = pack(e0, e1, T());
            }
            if (!CF::ALIAS) st16(tP + 16 * q, p);
          }
          const float2 sa = unpack2(sums[0]), sb = unpack2(sums[1]);
          sum = (sa.x + sa.y) + (sb.x + sb.y);
          const float mx = row_max();
          const bool over = mx > m + (HEADROOM<T> - START<T>) || (m == -INFINITY && mx != -INFINITY);
          if (!__any_sync(0xffffffffu, over)) break;
          // seldom: rescale to the new maximum (the scores' arrival says that the slot's last product is in) and again
          const float mn = over ? mx : m, f = m == -INFINITY ? (over ? 0.f : 1.f) : ex2(m - mn);
          m = mn;
          l *= f;
          if (any) {
#pragma unroll 1
            for (int j = 0; j < DH; j += 16) {
              uint32_t o[16];
              tc::ld16(tO + j, o);
#pragma unroll
              for (int u = 0; u < 16; ++u) o[u] = __float_as_uint(__uint_as_float(o[u]) * f);
              st16(tO + j, o);
            }
          }
        }
        any = true;
        l += sum;
        // (P of heads of 128 goes where the scores are, when they are no longer needed)
        if (CF::ALIAS) {
#pragma unroll
          for (int q = 0; q < C / 32; ++q) st16(tP + 16 * q, pk[q]);
        }
        st_wait();
        tc::fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(p_full + slot);
      }
      if (any) {
        const int last = steps - 1 - ((steps - 1 - k_first) & 1);
        ok = ok && wait(o_full + slot, ((g + last) >> 1) & 1);
        tc::fence_after();
      }
      g += steps;
      // ---- the rows' outputs: of two tiles each slot its own; of two shares each slot half the columns, out of both
      float f_mine = 1.f, f_other = 0.f;
      bool other = false;
      int j_lo = 0, j_hi = DH;
      if (!both) {
        s_ml[slot * 128 + i_row] = make_float2(m, l);
        tc::fence_before();
        sync();
        tc::fence_after();
        const float2 q = s_ml[(slot ^ 1) * 128 + i_row];
        other = steps > 1;                                   // (the other slot had a step)
        const float mm = fmaxf(m, q.x);
        // (no chunk on one side: maximum -inf and sum 0; a sum that is no number goes through)
        f_mine = !any ? 0.f : (m == -INFINITY ? 1.f : ex2(m - mm));
        f_other = !(other || !any) ? 0.f : (q.x == -INFINITY ? 1.f : ex2(q.x - mm));
        other = other || !any;
        l = (f_mine == 0.f ? 0.f : l * f_mine) + (f_other == 0.f ? 0.f : q.y * f_other);
        m = mm;
        j_lo = slot * (DH / 2); j_hi = j_lo + DH / 2;
      }
      const bool live = there && tree.reach[node][node >> 5] != 0u;
      const float inv = live ? 1.f / l : 0.f;
      const uint32_t tOther = tmem + CF::O_AT + (slot ^ 1) * DH + lanes;
      T* op = static_cast<T*>(a.out) + (int64_t)(s.r0 + node) * a.out_row + (hk * a.G + gh) * DH;
      float* part = a.part + ((size_t)(blockIdx.x * 2 + (w.starts() ? 1 : 0)) * 256 + (idx - w.mt * 256)) * (DH + 2);
#pragma unroll 1
      for (int j0 = j_lo; j0 < j_hi; j0 += 32) {
        uint32_t o[32];
        __syncwarp();
        if (any) {
          ld32(tO + j0, o);
          ld_wait();
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) o[j] = f_mine == 0.f ? 0u : __float_as_uint(__uint_as_float(o[j]) * f_mine);
        if (other) {
          uint32_t u[32];
          ld32(tOther + j0, u);
          ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (f_other != 0.f) o[j] = __float_as_uint(__uint_as_float(o[j]) + __uint_as_float(u[j]) * f_other);
        }
        if (*reinterpret_cast<volatile int*>(&s_bad) != 0 && there) {
          // values that are not finite, for the rows that see their key (p > 0)
          for (int c = w.c; c < w.c_end; ++c) {
            const Chunk ck = chunk_of<C>(s, c);
            if (!uneven_chunk<C>(a, s, ck)) continue;
            for (int k = 0; k < ck.n; ++k) {
              if (!((seen(a, tree, ck, node, depth, low, k & ~31) >> (k & 31)) & 1u)) continue;
              const T* v = values_of<T, DH>(a, s, ck, hk, k);
              if (v == nullptr) continue;
#pragma unroll
              for (int q = 0; q < 16; ++q) {
                const float2 u = unpack(reinterpret_cast<const uint32_t*>(v + j0)[q], T());
                if (!(fabsf(u.x) < INFINITY)) o[2 * q] = __float_as_uint(__uint_as_float(o[2 * q]) + u.x);
                if (!(fabsf(u.y) < INFINITY)) o[2 * q + 1] = __float_as_uint(__uint_as_float(o[2 * q + 1]) + u.y);
              }
            }
          }
        }
        if (!ok || !there) {
        } else if (whole) {
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            uint32_t p[4], q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {                    // (a row out of use: zeros, whatever the product holds)
              const float u = live ? __uint_as_float(o[j + 2 * k]) * inv : 0.f, v = live ? __uint_as_float(o[j + 2 * k + 1]) * inv : 0.f;
              p[k] = pack(u, v, T());
              q[k] = pack_rest(u, v, p[k]);
            }
            *reinterpret_cast<uint4*>(op + j0 + j) = make_uint4(p[0], p[1], p[2], p[3]);
            if (a.lo_off > 0) *reinterpret_cast<uint4*>(op + a.lo_off + j0 + j) = make_uint4(q[0], q[1], q[2], q[3]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 32; j += 2)
            *reinterpret_cast<float2*>(part + j0 + j) = live ? make_float2(__uint_as_float(o[j]), __uint_as_float(o[j + 1])) : make_float2(0.f, 0.f);
        }
      }
      if (ok && there && (both || slot == 0)) {
        if (!whole) *reinterpret_cast<float2*>(part + DH) = live ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
        else if (a.lse != nullptr) a.lse[(int64_t)(s.r0 + node) * a.H + hk * a.G + gh] = live ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
      }
      tc::fence_before();                                    // (O is read: the next tile's first product, behind p_full, may replace it)
      if (!both) sync();                                     // (by both slots' warps)
    }
    if (!ok) s_fail = 1;
  }
  __syncwarp();
  tc::fence_before();
  __syncthreads();
  tc::fence_after();
  if (s_fail) {                                              // a bounded wait gave up: report, once what was requested has landed
    if (threadIdx.x == 0 && a.status != nullptr) atomicMin(a.status, FM_ERR_TIMEOUT);
    ptx::drain_delay();
  }
  if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// ---- parts of the tiles that were cut, merged in order: grid (CTAs, blocks per tile); two, four or eight warps a row, by the number of
// parts (a tile has up to 148)
template <typename T, int DH, int ROWS>
__global__ void __launch_bounds__(256) merge_kernel(const __grid_constant__ Args a) {
  constexpr int CL = DH / 32, GS = ROWS * (DH + 2);
  __shared__ float s_o[8][DH];
  __shared__ float2 s_ml[8];
  ptx::grid_dep_wait();                                      // (dependents start at its end: blocks of the next pass beside these cost 5 us)
  const int4 d = __ldcg(a.desc + blockIdx.x);
  if (d.w < 2) return;
  const int r0 = a.row_off[d.x], n = min(a.row_off[d.x + 1] - r0, a.max_nodes), rows = min(ROWS, n * a.G - d.z * ROWS);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wpr = d.w <= 8 ? 2 : (d.w <= 32 ? 4 : 8), rpb = 8 / wpr, r = warp / wpr, q = warp - r * wpr;     // warps a row, rows a round
  for (int i0 = blockIdx.y * rpb; i0 < rows; i0 += gridDim.y * rpb) {
    const int i = i0 + r, idx = d.z * ROWS + i;
    const bool there = i < rows;
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
      const int per = (d.w + wpr - 1) / wpr, k1 = min(d.w, (q + 1) * per);     // neighbouring parts a warp
      for (int k0 = q * per; k0 < k1; k0 += U) {
        float2 ml[U];
        float v[U][CL];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = k0 + u;
          if (k >= k1) continue;
          const float* row = a.part + ((size_t)(blockIdx.x + k) * 2 + (k == 0 ? 1 : 0)) * GS + (size_t)i * (DH + 2);
          ml[u] = __ldcg(reinterpret_cast<const float2*>(row + DH));
#pragma unroll
          for (int j = 0; j < CL; ++j) v[u][j] = __ldcg(row + lane + 32 * j);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k0 + u < k1) add(ml[u].x, ml[u].y, v[u]);
      }
    }
    __syncthreads();                                         // (the rows before have been read)
    if (q != 0) {
#pragma unroll
      for (int j = 0; j < CL; ++j) s_o[warp][lane + 32 * j] = o[j];
      if (lane == 0) s_ml[warp] = make_float2(m, l);
    }
    __syncthreads();
    if (q != 0 || !there) continue;
    for (int k = 1; k < wpr; ++k) {
      float o2[CL];
#pragma unroll
      for (int j = 0; j < CL; ++j) o2[j] = s_o[warp + k][lane + 32 * j];
      add(s_ml[warp + k].x, s_ml[warp + k].y, o2);
    }
    const int nd = a.g_div(idx), gh = idx - nd * a.G, h = d.y * a.G + gh;
    const bool live = !(m == -INFINITY && l == 0.f);         // (a node in use sees itself)
    const float inv = live ? 1.f / l : 0.f;
    T* out = static_cast<T*>(a.out) + (int64_t)(r0 + nd) * a.out_row + (int64_t)h * DH;
#pragma unroll
    for (int j = 0; j < CL; ++j) {
      const uint32_t hi = pack(o[j] * inv, 0.f, T());
      reinterpret_cast<unsigned short*>(out)[lane + 32 * j] = (unsigned short)hi;
      if (a.lo_off > 0) reinterpret_cast<unsigned short*>(out)[a.lo_off + lane + 32 * j] = (unsigned short)pack_rest(o[j] * inv, 0.f, hi);
    }
    if (lane == 0 && a.lse != nullptr) a.lse[(int64_t)(r0 + nd) * a.H + h] = live ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  }
}

// ------------------------------------------------------------------------------------------
// the longest confirmed path: a warp per tree, eight nodes a lane
// ------------------------------------------------------------------------------------------
// By a warp: calls put(i, node) in lane 0 for the nodes of the path, returns their number; `next`: the prediction at the last one.
template <typename Put>
__device__ inline int walk_path(const int* tokens, const int* parent, const int* predicted, int n, int lane, int& next, Put put) {
  constexpr int PER = FM_MAX_TREE_NODES / 32;
  int par[PER], tok[PER], pre[PER];
  n = min(n, FM_MAX_TREE_NODES);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int i = k * 32 + lane;
    par[k] = i < n ? parent[i] : -2;
    tok[k] = i < n ? tokens[i] : 0;
    pre[k] = i < n ? predicted[i] : 0;
  }
  int cur = n > 0 && __shfl_sync(0xffffffffu, par[0], 0) == -1 ? 0 : -1, at = 0;
  while (cur >= 0) {                                         // (every step goes to a later node)
    if (lane == 0) put(at, cur);
    ++at;
    int mine = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) if ((cur >> 5) == k) mine = pre[k];
    next = __shfl_sync(0xffffffffu, mine, cur & 31);
    int child = -1;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const unsigned hit = __ballot_sync(0xffffffffu, par[k] == cur && tok[k] == next && k * 32 + lane > cur);
      if (child < 0 && hit != 0) child = k * 32 + __ffs(hit) - 1;
    }
    cur = child;
  }
  return at;
}
static __global__ void __launch_bounds__(128) accept_kernel(const int* tokens, const int* parent, const int* row_off, const int* predicted, int batch,
                                                     int rows, int* path, int path_stride, int* n_acc, int* next_tok) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= batch) return;
  const int from = row_off[b], end = row_off[b + 1];
  const bool none = from < 0 || end < from || end > rows;    // not rows that there are
  const int r0 = none ? 0 : from, n = none ? 0 : min(end - from, path_stride);
  int next = -1;
  const int at = walk_path(tokens + r0, parent + r0, predicted + r0, n, lane, next, [&](int i, int node) { path[(int64_t)b * path_stride + i] = node; });
  for (int j = at + lane; j < path_stride; j += 32) path[(int64_t)b * path_stride + j] = -1;
  if (lane == 0) { n_acc[b] = at; next_tok[b] = at > 0 ? next : -1; }
}

constexpr size_t DESC_BYTES = 8192;      // in front of a workspace's parts: what the merge has to do, of the CTAs
// Launches, for the entry points and for the context's own passes (fm_ops.cu).
size_t workspace_bytes(int max_nodes, int group, int head_dim);
bool make_maps(const fm_cache& c, int layer, int max_pages, Args& a);          // the sizes in `a` are set
int launch(const Args& a, int dtype, int head_dim, cudaStream_t stream);
int launches(const Args& a, int head_dim);                   // of kernels, by that: two where a tile may be cut
Div div_by(int d);

}  // namespace tr
