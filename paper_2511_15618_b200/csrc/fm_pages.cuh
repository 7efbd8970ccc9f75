// Pages of a shared cache pool: hand out, share, copy on write, give back, compact; rows appended behind a sequence.
//
// The bookkeeping is integers in device memory, so that a decode loop never waits for the host: fork and truncate are
// one block per entry, reserve and compact plan in one block (prefix sums over the entries and over the free pages, in
// id order, so the result does not depend on timing) and a second launch moves the data.  Launches of a decode loop follow one
// another on a stream: each is already resident when the one in front ends.
// Moving is bound by memory: 16-byte loads and stores, a block per (page or rows, layer, key or value): pages of their own for 96 forks
// of 16 sequences in 32 layers and a row behind each, 834 MB: 104 us (partly from L2); compaction of 1.5 GB: 267 us, 5.7 TB/s (87 % of a copy).
// Small calls are the latency of the planning chain (lengths, tables, references, free list): 5 to 7 us.
#pragma once
#include "fm_common.cuh"
#include "fm_ptx.cuh"
#include "../../include/flashmesh.h"

namespace pg {

constexpr int PLAN = 1024;              // threads of a planning block
constexpr int PER = FM_MAX_SEQS / PLAN; // entries per thread of it

struct Geo {                            // one of the pool's two halves is chosen by the block
  char *k, *v;
  int64_t layer, page, head, slot;      // bytes
  int layers, heads, row16;             // 16-byte pieces of a head's row
};

// work: [0, n_pages) list A, [n_pages, 2 n_pages) list B, then copy jobs (old, new, slots) of the entries, counters of the
// entries, and one word
__host__ __device__ inline int64_t jobs_at(const fm_pages& p) { return 2 * (int64_t)p.n_pages; }
__host__ __device__ inline int64_t counters_at(const fm_pages& p) { return jobs_at(p) + 3 * (int64_t)p.max_seqs; }
__host__ __device__ inline int64_t word_at(const fm_pages& p) { return counters_at(p) + p.max_seqs; }

__device__ inline void fail(const fm_pages& p, int code) { atomicMin(p.status, code); }
__device__ inline int pages_of(int slots, int page_slots) { return slots <= 0 ? 0 : (slots - 1) / page_slots + 1; }
__device__ inline bool page_ok(const fm_pages& p, int id) { return id >= 0 && id < p.n_pages; }
__device__ inline int len_of(const fm_pages& p, int seq) {           // what the table can hold, whatever stands there
  const int64_t most = (int64_t)p.max_pages * p.page_slots;
  const int n = p.lens[seq];
  return n < 0 ? 0 : (n > most ? (int)most : n);
}

__global__ void reset_kernel(const fm_pages p) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, stride = (int64_t)gridDim.x * blockDim.x;
  for (int64_t j = i; j < (int64_t)p.max_seqs * p.max_pages; j += stride) p.table[j] = -1;
  for (int64_t j = i; j < p.max_seqs; j += stride) p.lens[j] = 0;
  for (int64_t j = i; j < p.n_pages; j += stride) p.refs[j] = 0;
  for (int64_t j = i; j <= word_at(p); j += stride) p.work[j] = 0;
  if (i == 0) *p.status = 0;
}

// Is entry e of a list usable?  0: yes, 1: skip it silently, 2: a bad or repeated id.  Called by a whole block.
__device__ inline int entry_state(const int* ids, int e, int limit) {
  const int id = ids[e];
  int twice = 0;
  if (id >= 0 && id < limit)
    for (int j = threadIdx.x; j < e; j += blockDim.x) twice |= ids[j] == id;
  twice = __syncthreads_or(twice);
  return id < 0 ? 1 : (id >= limit || twice ? 2 : 0);
}

// ---- fork: a block per entry.  No source of the call is a destination of it, so tables read here are not written here.
__global__ void fork_kernel(const fm_pages p, const int* src, const int* dst, int n) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int e = blockIdx.x, s = src[e], d = dst[e];
  if (s < 0 || d < 0) return;
  int bad = s >= p.max_seqs || d >= p.max_seqs;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    const int sj = src[j], dj = dst[j];
    if (sj < 0) continue;
    bad |= dj == s || (j < e && dj == d);
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) fail(p, FM_ERR_INVALID_ARG);
    return;
  }
  const int len = len_of(p, s), held = pages_of(len, p.page_slots);
  int* to = p.table + (int64_t)d * p.max_pages;
  const int* from = p.table + (int64_t)s * p.max_pages;
  for (int j = threadIdx.x; j < p.max_pages; j += blockDim.x) {
    const int old = to[j], id = j < held ? from[j] : -1;
    if (page_ok(p, id)) atomicAdd(p.refs + id, 1);
    if (page_ok(p, old)) atomicSub(p.refs + old, 1);
    if (old != id) to[j] = id;
  }
  if (threadIdx.x == 0) p.lens[d] = len;
}

// ---- truncate: a block per entry
__global__ void truncate_kernel(const fm_pages p, const int* seqs, const int* new_lens) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int e = blockIdx.x, state = entry_state(seqs, e, p.max_seqs);
  if (state != 0) {
    if (state == 2 && threadIdx.x == 0) fail(p, FM_ERR_INVALID_ARG);
    return;
  }
  const int s = seqs[e], left = min(len_of(p, s), max(new_lens[e], 0));
  __syncthreads();                                           // the length has been read
  int* t = p.table + (int64_t)s * p.max_pages;
  for (int j = pages_of(left, p.page_slots) + threadIdx.x; j < p.max_pages; j += blockDim.x) {
    const int id = t[j];
    if (page_ok(p, id)) atomicSub(p.refs + id, 1);
    if (id != -1) t[j] = -1;
  }
  if (threadIdx.x == 0) p.lens[s] = left;
}

// exclusive prefix sum over the block's threads; the total in every thread
__device__ inline int block_scan(int v, int* sh, int& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) sh[w] = x;
  __syncthreads();
  int y = sh[lane];                                          // PLAN / 32 = 32 warps
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  total = __shfl_sync(0xffffffffu, y, 31);
  const int before = __shfl_sync(0xffffffffu, y, (w + 31) & 31);
  return (w == 0 ? 0 : before) + x - v;
}

// ---- reserve, planning: one block
__global__ void __launch_bounds__(PLAN) reserve_plan_kernel(const fm_pages p, const int* seqs, const int* grow, int n) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  __shared__ int s_seq[FM_MAX_SEQS], s_held[FM_MAX_SEQS];    // sequence or -1; partly filled last page that is to grow, or -1
  __shared__ int sh[32];
  int* list = p.work;                                        // free ids, lowest first
  int* jobs = p.work + jobs_at(p);
  for (int e = threadIdx.x; e < n; e += PLAN) s_seq[e] = seqs[e];
  __syncthreads();
  // What every entry wants.  Entries of a thread: e = PER * thread + i would be uneven for short lists; the prefix sum
  // runs round by round instead (a round: PLAN entries in order).
  int want[PER], first[PER], len[PER];
  bool cow[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * PLAN + threadIdx.x;
    want[i] = 0; first[i] = 0; len[i] = 0; cow[i] = false;
    if (e < n) {
      int s = s_seq[e], held = -1;
      if (s >= 0) {
        bool bad = s >= p.max_seqs;
        for (int j = 0; j < e && !bad; ++j) bad = s_seq[j] == s;
        const int g = bad ? 0 : max(grow[e], 0);
        if (bad) {
          fail(p, FM_ERR_INVALID_ARG);
        } else if (g > 0) {
          len[i] = len_of(p, s);
          const int64_t end = (int64_t)len[i] + g;
          if (end > (int64_t)p.max_pages * p.page_slots) {
            fail(p, FM_ERR_CAPACITY);
          } else {
            const int* t = p.table + (int64_t)s * p.max_pages;
            const int need = pages_of((int)end, p.page_slots);
            int have = pages_of(len[i], p.page_slots);
            while (have < need && page_ok(p, t[have])) ++have;
            first[i] = have;
            want[i] = need - have;
            if (len[i] % p.page_slots != 0 && page_ok(p, t[len[i] / p.page_slots])) held = t[len[i] / p.page_slots];
          }
        }
      }
      s_held[e] = held;
    }
  }
  __syncthreads();
  int total = 0, at[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * PLAN + threadIdx.x;
    at[i] = 0;
    if (i * PLAN >= n) continue;
    if (e < n && s_held[e] >= 0) {
      const int held = s_held[e];
      int before = 0;                                        // entries in front that leave the same page
      for (int j = 0; j < e; ++j) before += s_held[j] == held;
      cow[i] = p.refs[held] - before > 1;
      want[i] += cow[i] ? 1 : 0;
    }
    int t;
    at[i] = total + block_scan(e < n ? want[i] : 0, sh, t);
    total += t;
  }
  // Tables that could ask for 2^31 pages in one call: the sum may have left 32 bits.  All free pages are listed, and handed out entry by entry.
  if ((int64_t)n * ((int64_t)p.max_pages + 1) > INT_MAX) total = INT_MAX;
  // the lowest `total` free ids
  int found = 0;
  for (int64_t p0 = 0; p0 < p.n_pages && found < total; p0 += 4 * PLAN) {
    int r[4], mine = 0;
    const int64_t base = p0 + 4 * threadIdx.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) { r[j] = base + j < p.n_pages ? p.refs[base + j] : 1; mine += r[j] <= 0; }
    int t, to = found + block_scan(mine, sh, t);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (r[j] <= 0) list[to++] = (int)(base + j);
    found += t;
  }
  __syncthreads();
  if (found < total) {                                       // not for all (or too many to add up): entry by entry, in order
    if (threadIdx.x != 0) return;
    int next = 0;
    for (int e = 0; e < n; ++e) {
      jobs[3 * e] = -1;
      const int s = s_seq[e];
      bool ok = s >= 0 && s < p.max_seqs && grow[e] > 0;
      for (int j = 0; j < e && ok; ++j) ok = s_seq[j] != s;
      if (!ok) continue;
      const int l = len_of(p, s), held = s_held[e];
      const int64_t end = (int64_t)l + grow[e];
      if (end > (int64_t)p.max_pages * p.page_slots) continue;
      int* t = p.table + (int64_t)s * p.max_pages;
      const int need = pages_of((int)end, p.page_slots);
      int have = pages_of(l, p.page_slots);
      while (have < need && page_ok(p, t[have])) ++have;
      const bool copy = held >= 0 && p.refs[held] > 1;
      if (need - have + (copy ? 1 : 0) > found - next) { fail(p, FM_ERR_CAPACITY); continue; }
      if (copy) {
        const int id = list[next++];
        jobs[3 * e] = held; jobs[3 * e + 1] = id; jobs[3 * e + 2] = l % p.page_slots;
        p.refs[held] -= 1;
        p.refs[id] = 1;
        t[l / p.page_slots] = id;
      }
      for (int j = have; j < need; ++j) { const int id = list[next++]; p.refs[id] = 1; t[j] = id; }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = i * PLAN + threadIdx.x;
    if (e >= n) continue;
    int from = at[i];
    jobs[3 * e] = cow[i] ? s_held[e] : -1;
    if (want[i] == 0) continue;
    int* t = p.table + (int64_t)s_seq[e] * p.max_pages;
    if (cow[i]) {
      const int id = list[from++];
      jobs[3 * e + 1] = id; jobs[3 * e + 2] = len[i] % p.page_slots;
      atomicSub(p.refs + s_held[e], 1);
      p.refs[id] = 1;
      t[len[i] / p.page_slots] = id;
    }
    const int more = want[i] - (cow[i] ? 1 : 0);
    for (int j = 0; j < more; ++j) { const int id = list[from + j]; p.refs[id] = 1; t[first[i] + j] = id; }
  }
}

// rows [0, slots) of every head of a page -> another page; by a block, U pieces of a thread under way: 4 for parts of pages just
// written or read (96 forks, 32 layers: 104 us; 8: 122, 1: 131), 8 for whole pages of a pool (1.5 GB: 267 us; 4: 277, 1: 287)
template <int U>
__device__ inline void copy_page(const Geo& g, char* base, int from, int to, int slots) {
  const int per = slots * g.row16, all = g.heads * per;
  const char* src = base + from * g.page;
  char* dst = base + to * g.page;
  for (int i0 = threadIdx.x; i0 < all; i0 += U * blockDim.x) {
    int64_t at[U];
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * blockDim.x, h = i / per, r = i - h * per, s = r / g.row16, c = r - s * g.row16;
      at[u] = h * g.head + s * g.slot + 16 * c;
      if (i < all) x[u] = *reinterpret_cast<const uint4*>(src + at[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * (int)blockDim.x < all) *reinterpret_cast<uint4*>(dst + at[u]) = x[u];
  }
}

// ---- reserve, copies of shared pages: grid (entries, layers * 2)
__global__ void __launch_bounds__(256) reserve_copy_kernel(const fm_pages p, const Geo g) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int* job = p.work + jobs_at(p) + 3 * blockIdx.x;
  const int old = __ldcg(job);
  if (old < 0) return;
  char* base = ((blockIdx.y & 1) ? g.v : g.k) + (blockIdx.y >> 1) * g.layer;
  copy_page<4>(g, base, old, __ldcg(job + 1), __ldcg(job + 2));
}

// ---- append: grid (entries, blocks of an entry); the last block of an entry advances the length.  A block checks the entry (a chain of six
// dependent reads) and moves its share of the layers' keys and values, four at a time: with a block for each, forks, copies and rows of
// 96 entries in 32 layers took 147 us in place of 131 (before pages were copied four pieces at a time).
struct Rows {
  const char *k, *v;
  int64_t layer, row, head;             // bytes
  int n_rows;                           // rows that there are, 0: not said
};
__global__ void __launch_bounds__(256) append_kernel(const fm_pages p, const Geo g, const Rows rows, const int* seqs, const int* row_off,
                                                     const int* path, int path_stride, const int* n_acc, int max_rows) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int e = blockIdx.x, s = seqs[e], r0 = row_off[e], end = row_off[e + 1], own = r0 >= 0 && end > r0 ? end - r0 : 0;
  const int n = max(path != nullptr ? n_acc[e] : own, 0);
  const int state = entry_state(seqs, e, p.max_seqs);
  if (state != 0) {
    if (state == 2 && threadIdx.x == 0 && blockIdx.y == 0) fail(p, FM_ERR_INVALID_ARG);
    return;
  }
  const int len = len_of(p, s);
  const int* t = p.table + (int64_t)s * p.max_pages;
  // all or nothing: the pages are there and the sequence's own, the rows are its rows
  int bad = 0;
  if (n > max_rows || r0 < 0 || (rows.n_rows > 0 && end > rows.n_rows) || (path != nullptr && n > path_stride)) bad = 1;
  else if ((int64_t)len + n > (int64_t)p.max_pages * p.page_slots) bad = 2;
  else {
    if (path != nullptr)
      for (int j = threadIdx.x; j < n; j += blockDim.x) { const int r = path[(int64_t)e * path_stride + j]; if (r < 0 || r >= own) bad |= 1; }
    for (int j = len / p.page_slots + threadIdx.x; n > 0 && j < pages_of(len + n, p.page_slots); j += blockDim.x)
      if (!page_ok(p, t[j]) || p.refs[t[j]] != 1) bad |= 2;
  }
  const int wrong = __syncthreads_or(bad & 1), missing = __syncthreads_or(bad & 2);
  if (!wrong && !missing) {
    // a piece lies at the same place in every layer's keys and values; threads share the layers where there are few pieces
    const int per = g.heads * g.row16, pieces = n * per;
    int wide = 256;
    while (wide > 32 && wide / 2 >= pieces) wide /= 2;
    const int first = blockIdx.y + gridDim.y * (threadIdx.x / wide), step = gridDim.y * (256 / wide);
    for (int i = threadIdx.x & (wide - 1); i < pieces; i += wide) {
      const int j = i / per, r = i - j * per, h = r / g.row16, c = r - h * g.row16;
      const int row = r0 + (path != nullptr ? path[(int64_t)e * path_stride + j] : j), at = len + j, pi = at / p.page_slots;
      const int64_t from = row * rows.row + h * rows.head + 16 * c, to = t[pi] * g.page + h * g.head + (at - pi * p.page_slots) * g.slot + 16 * c;
      for (int l0 = first; l0 < 2 * g.layers; l0 += 4 * step) {
        uint4 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int l = l0 + u * step;
          if (l < 2 * g.layers) x[u] = *reinterpret_cast<const uint4*>(((l & 1) ? rows.v : rows.k) + (l >> 1) * rows.layer + from);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int l = l0 + u * step;
          if (l < 2 * g.layers) *reinterpret_cast<uint4*>(((l & 1) ? g.v : g.k) + (l >> 1) * g.layer + to) = x[u];
        }
      }
    }
  } else if (threadIdx.x == 0 && blockIdx.y == 0) {
    fail(p, wrong ? FM_ERR_INVALID_ARG : FM_ERR_BAD_STATE);
  }
  // (every block of the entry has read the length when the counter is full; it wraps to zero for the next call)
  __syncthreads();
  if (threadIdx.x == 0) {
    const unsigned seen = atomicInc(reinterpret_cast<unsigned*>(p.work + counters_at(p) + e), gridDim.y - 1);
    if (seen == gridDim.y - 1 && !wrong && !missing) p.lens[s] = len + n;
  }
}

// ---- compact, planning: one block.  Sources all lie at or behind `used`, destinations in front of it: no page is both.
__global__ void __launch_bounds__(PLAN) compact_plan_kernel(const fm_pages p, int* used) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  __shared__ int sh[32];
  int count = 0, n_used;
  for (int64_t i = threadIdx.x; i < p.n_pages; i += PLAN) count += p.refs[i] > 0;
  block_scan(count, sh, n_used);
  int *holes = p.work, *goes = p.work + p.n_pages;           // goes: page behind `used` -> its index among the movers
  int n_holes = 0, n_movers = 0;
  for (int64_t p0 = 0; p0 < p.n_pages; p0 += 4 * PLAN) {
    int r[4], h = 0, m = 0;
    const int64_t base = p0 + 4 * threadIdx.x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r[j] = base + j < p.n_pages ? p.refs[base + j] : -1;
      if (base + j < p.n_pages && base + j < n_used) h += r[j] <= 0;
      if (base + j >= n_used) m += r[j] > 0;
    }
    int th, tm, ah = n_holes + block_scan(h, sh, th), am = n_movers + block_scan(m, sh, tm);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t i = base + j;
      if (i >= p.n_pages) continue;
      if (i < n_used && r[j] <= 0) holes[ah++] = (int)i;
      if (i >= n_used && r[j] > 0) { holes[p.n_pages - 1 - am] = (int)i; goes[i] = am++; }   // movers from the end of the list
    }
    n_holes += th;
    n_movers += tm;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < n_movers; k += PLAN) {
    const int from = holes[p.n_pages - 1 - k], to = holes[k];
    p.refs[to] = p.refs[from];
    p.refs[from] = 0;
  }
  if (threadIdx.x == 0) {
    p.work[word_at(p)] = n_movers;
    if (used != nullptr) *used = n_used;
  }
}

// grid (blocks, layers * 2 + 1): the last row of blocks rewrites the tables
__global__ void __launch_bounds__(256) compact_copy_kernel(const fm_pages p, const Geo g) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int n = __ldcg(p.work + word_at(p));
  const int *list = p.work, *goes = p.work + p.n_pages;
  if ((int)blockIdx.y == 2 * g.layers) {
    if (n == 0) return;
    // pages in front of the pages in use keep their ids; the first mover is the lowest id that does not
    const int first = __ldcg(list + p.n_pages - 1);
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)p.max_seqs * p.max_pages; i += (int64_t)gridDim.x * blockDim.x) {
      const int id = p.table[i];
      if (id < first || id >= p.n_pages) continue;
      const unsigned k = (unsigned)__ldcg(goes + id);
      if (k < (unsigned)n && __ldcg(list + p.n_pages - 1 - k) == id) p.table[i] = __ldcg(list + k);
    }
    return;
  }
  char* base = ((blockIdx.y & 1) ? g.v : g.k) + (blockIdx.y >> 1) * g.layer;
  for (int k = blockIdx.x; k < n; k += gridDim.x)
    copy_page<8>(g, base, __ldcg(list + p.n_pages - 1 - k), __ldcg(list + k), p.page_slots);
}

}  // namespace pg
