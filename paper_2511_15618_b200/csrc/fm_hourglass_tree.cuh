// A tree of candidates through the hourglass: rows and parents of every level, the row-wise pieces between the level
// stacks, and what moves an accepted path into the caches and carry rings.
//
// A node of the tree is a coordinate position L + depth.  Where that is a multiple of three it is also a vertex row, where
// it is a multiple of nine a face row; a row's parent at its level is the nearest ancestor that has one.  Level rows of a
// sequence are numbered in the order of their nodes (a parent's is lower), rows b * N + i, the rest of the N unused.
// Keys and values of the nodes stay in buffers of their own until a path is accepted: nothing of the caches or rings
// changes before, and siblings never share a slot.
#pragma once
#include "fm_kernels.cuh"
#include "fm_tree.cuh"

namespace ht {

struct Tree {
  int N;                                // rows per sequence at every level
  PackedRow* row[3];                    // [B * N] sequence (-1: unused), level-local position, -, cache slot behind the prefix
  int* par[3];                          // [B * N] parent: row of the sequence, -1: continues the cache, -2: unused
  int* node[3];                         // [B * N] the row's node
  int* low[2];                          // [B * N][3] rows (of all) of the level below that a vertex / face row pools, -1: from the ring or nothing
  int* up[2];                           // [B * N] row of the level above a coordinate / vertex row belongs to, -1: from the ring
  int *off, *len[3], *ident;            // [B + 1] row offsets, [B] cached slots (prefix included) per level, [B] 0, 1, ...
  int *tok, *pred, *acc;                // [B * N] tokens, predictions, accepted (1) or not
  float *h[2], *tri[2], *z[3];          // pre-shorten hiddens (coordinate, vertex), upsampled triples (of vertices, of faces), inputs of the last layers
  bf16 *k, *v;                          // [layers][rows][Hkv * dh]
  int rows_alloc;
};

// A thread per sequence: a tree has at most 28 nodes, one after the other: each needs its parent's entries.
static __global__ void map_kernel(Dims dm, SeqState st, Tree t, const int* parent, int batch) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b > batch) return;
  t.off[b] = b * t.N;
  if (b == batch) return;
  const int N = t.N, L = st.L[b], most = st.nrow[b];
  const int* p = parent + (size_t)b * N;
  int n[3] = {0, 0, 0}, pos[FM_MAX_DRAFT + 1], at[3][FM_MAX_DRAFT + 1];        // position (-1: unused) and level rows of a node, or of its nearest ancestor
  t.ident[b] = b;
  for (int l = 0; l < 3; ++l) {
    const int r = fm_ratio(l);
    t.len[l][b] = dm.P + (L + r - 1) / r;
  }
  for (int i = 0; i < N; ++i) {
    const int q = p[i], base = b * N;
    const bool root = i == 0 && q == -1, child = q >= 0 && q < i && pos[q] >= 0;
    pos[i] = root ? L : (child ? pos[q] + 1 : -1);
    if (pos[i] - L >= most) pos[i] = -1;                     // (no row of this depth is fed any more)
    const int P = pos[i];
    for (int l = 0; l < 3; ++l) {
      const int r = fm_ratio(l), above = root ? -1 : (child ? at[l][q] : -1);
      at[l][i] = above;
      if (P < 0 || (l > 0 && P % r != 0)) continue;
      const int row = l == 0 ? i : n[l];
      n[l] = l == 0 ? i + 1 : n[l] + 1;
      t.row[l][base + row] = PackedRow{b, P / r, 0, (P / r) % dm.cap[l]};
      t.par[l][base + row] = above;
      t.node[l][base + row] = i;
      at[l][i] = row;
    }
    if (P < 0) {
      t.row[0][base + i] = PackedRow{-1, 0, 0, 0};
      t.par[0][base + i] = -2;
      t.node[0][base + i] = i;
    }
    // the row above: the nearest ancestor's, where that is the position's own vertex (face)
    if (P >= 0) t.up[0][base + i] = at[1][i] >= 0 && t.row[1][base + at[1][i]].p == P / 3 ? base + at[1][i] : -1;
  }
  for (int l = 1; l < 3; ++l) {
    for (int i = n[l]; i < N; ++i) {
      t.row[l][b * N + i] = PackedRow{-1, 0, 0, 0};
      t.par[l][b * N + i] = -2;
      t.node[l][b * N + i] = -1;
    }
    for (int i = 0; i < n[l]; ++i) {
      // its own row below and that row's two ancestors; those in front of the pass are in the ring
      int low = l == 1 ? t.node[1][b * N + i] : at[1][t.node[2][b * N + i]];
      for (int k = 2; k >= 0; --k) {
        t.low[l - 1][3 * (b * N + i) + k] = low >= 0 ? b * N + low : -1;
        if (low >= 0) low = t.par[l - 1][b * N + low];
      }
    }
  }
  for (int i = 0; i < n[1]; ++i) {
    const int f = at[2][t.node[1][b * N + i]], v = t.row[1][b * N + i].p;
    t.up[1][b * N + i] = f >= 0 && t.row[2][b * N + f].p == v / 3 ? b * N + f : -1;
  }
}

static __global__ void embed_kernel(Dims dm, SeqState st, Tree t, const int* tokens, const bf16* __restrict__ E, float* __restrict__ x,
                                    const float* __restrict__ g, bf16* __restrict__ a, float* __restrict__ ssq, int ld_ssq) {
  const int row = blockIdx.x;
  const PackedRow r = t.row[0][row];
  int tok = tokens[row];
  if (threadIdx.x == 0) t.tok[row] = tok;
  if (r.b >= 0 && (tok < 0 || tok >= dm.V || (row % t.N == 0 && tok != st.main_tok[r.b]))) {
    if (threadIdx.x == 0) atomicExch(st.status, -1);
    if (tok < 0 || tok >= dm.V) tok = dm.n_bins + 2;         // never index outside the table
  }
  for (int i = threadIdx.x; i < dm.d; i += blockDim.x) x[(size_t)row * dm.d + i] = r.b >= 0 ? __bfloat162float(E[(size_t)tok * dm.d + i]) : 0.f;
  __syncthreads();
  stack_entry_row(x + (size_t)row * dm.d, row, dm.d, g, a, ssq, ld_ssq);
}

// operand rows of a shorten GEMM; grid (rows, 3)
static __global__ void gather_kernel(Dims dm, Tree t, int lu, const float* x_low, const float* ring, bf16* __restrict__ out) {
  const int row = blockIdx.x, part = blockIdx.y, d = dm.d, rs = fm_ring(lu - 1);
  const PackedRow r = t.row[lu][row];
  const int pos = 3 * r.p - 2 + part, low = r.b >= 0 ? t.low[lu - 1][3 * row + part] : -1;
  const float* src = low >= 0 ? x_low + (size_t)low * d : ring + ((size_t)max(r.b, 0) * rs + ((pos + rs) % rs)) * d;
  const bool ok = r.b >= 0 && pos >= 0;
  for (int i = threadIdx.x; i < d; i += blockDim.x) store_hi_lo(out + (size_t)row * 6 * d + part * d + i, ok ? src[i] : 0.f, 3 * d);
}

// x (the pre-shorten hidden, kept in h) += the row's slot of the triple above
static __global__ void upsample_kernel(Dims dm, Tree t, int level, const float* tri_ring, float* __restrict__ x, const float* __restrict__ g,
                                       bf16* __restrict__ a, float* __restrict__ ssq, int ld_ssq) {
  const int row = blockIdx.x, d = dm.d, rsu = fm_ring(level + 1);
  const PackedRow r = t.row[level][row];
  const int up = r.b >= 0 ? t.up[level][row] : -1;
  const float* s = (up >= 0 ? t.tri[level] + (size_t)up * 3 * d : tri_ring + ((size_t)max(r.b, 0) * rsu + (r.p / 3) % rsu) * 3 * d) + (r.p % 3) * d;
  float *xr = x + (size_t)row * d, *hr = t.h[level] + (size_t)row * d;
  for (int i = threadIdx.x; i < d; i += blockDim.x) {
    const float v = xr[i];
    hr[i] = v;
    xr[i] = r.b >= 0 ? v + s[i] : 0.f;
  }
  __syncthreads();
  stack_entry_row(xr, row, d, g, a, ssq, ld_ssq);
}

// masked argmax of every node's logits, as verify_top2_kernel's
static __global__ void top_kernel(Dims dm, Tree t, const float* logits, float* __restrict__ logits_out, int* __restrict__ out, float* __restrict__ margin_out) {
  const int row = blockIdx.x;
  const PackedRow r = t.row[0][row];
  if (logits_out != nullptr)
    for (int i = threadIdx.x; i < dm.V; i += blockDim.x) logits_out[(size_t)row * dm.V + i] = r.b >= 0 ? logits[(size_t)row * dm.Vpad + i] : 0.f;
  Top2 q{0.f, -1, 0.f};
  if (r.b >= 0) q = block_top2(logits + (size_t)row * dm.Vpad, dm, r.p);
  if (threadIdx.x == 0) {
    t.pred[row] = q.i1;
    if (out != nullptr) out[row] = q.i1;
    if (margin_out != nullptr) margin_out[row] = r.b >= 0 ? q.v1 - q.v2 : 0.f;
  }
}

// acceptance: the walk of fm_tree_accept, then what accept_one does with an accepted run.  One block.
static __global__ void accept_kernel(Dims dm, SeqState st, Tree t, int batch, const int* force_pred, int* __restrict__ path, int* __restrict__ n_acc,
                                     int* __restrict__ emitted, int* __restrict__ kv_len) {
  const int lane = threadIdx.x & 31, N = t.N, eos = dm.n_bins + 1;
  for (int b = threadIdx.x >> 5; b < batch; b += blockDim.x >> 5) {
    const int base = b * N;
    for (int i = lane; i < N; i += 32) {
      t.acc[base + i] = 0;
      if (path != nullptr) path[base + i] = -1;
      if (emitted != nullptr) emitted[base + i] = -1;
    }
    __syncwarp();
    const int L = st.L[b], rows = st.nrow[b];                // (rows: the limits may have changed since the tree was verified)
    int next = 0, a = 0, last = 0;
    bool fin = false;
    const int* pred = force_pred != nullptr ? force_pred + base : t.pred + base;
    if (rows > 0 && !st.done[b]) {
      a = tr::walk_path(t.tok + base, t.par[0] + base, pred, N, lane, next, [&](int i, int node) {
        if (fin || i >= rows) return;                        // (lane 0: behind an accepted EOS, or the last position; the next token is none's then)
        const int tok = t.tok[base + node];
        t.acc[base + node] = 1;
        st.hist[b * FM_HIST + ((L - 1 + i) & (FM_HIST - 1))] = tok;
        if (path != nullptr) path[base + i] = node;
        if (emitted != nullptr) emitted[base + i] = tok;
        last = i + 1;
        fin = tok == eos;
      });
      a = __shfl_sync(0xffffffffu, last, 0);
      fin = __shfl_sync(0xffffffffu, (int)fin, 0) != 0;
      if (lane == 0 && a > 0) {
        if (L + a - 1 >= st.t_end[b]) fin = true;
        st.L[b] = L + a;
        st.main_tok[b] = next;
        st.done[b] = fin ? 1 : 0;
        st.nrow[b] = fin ? 0 : min(dm.R1, st.t_end[b] - (L + a - 1));
      }
    } else if (lane == 0) {
      st.nrow[b] = 0;
    }
    if (lane == 0) {
      if (n_acc != nullptr) n_acc[b] = a;
      if (kv_len != nullptr) { kv_len[b * 3] = L + a; kv_len[b * 3 + 1] = (L + a + 2) / 3; kv_len[b * 3 + 2] = (L + a + 8) / 9; }
    }
  }
  __syncthreads();
  count_rows(dm, st, batch);
}

// keys, values, hiddens, triples and split nodes of the accepted rows to where the next pass looks for them; grid (rows,
// layers + 3)
template <typename LayerPtr>
static __global__ void commit_kernel(Dims dm, Tree t, const LayerPtr* __restrict__ layers, int n_layers, float* hc_ring, float* hv_ring, float* trif_ring,
                                     float* triv_ring, float* zc, float* zv, float* zf) {
  const int row = blockIdx.x, y = blockIdx.y, d = dm.d, kvw = dm.Hkv * dm.dh;
  const int l = y < n_layers ? layers[y].level : y - n_layers;
  const PackedRow r = t.row[l][row];
  if (r.b < 0 || t.acc[r.b * t.N + t.node[l][row]] == 0) return;
  if (y < n_layers) {
    const int slots = dm.P + dm.cap[l];
    const size_t from = ((size_t)y * t.rows_alloc + row) * kvw;
    for (int i = threadIdx.x; i < kvw / 8; i += blockDim.x) {
      const int hk = 8 * i / dm.dh, c = 8 * i - hk * dm.dh;
      const size_t to = (((size_t)r.b * dm.Hkv + hk) * slots + dm.P + r.slot) * dm.dh + c;
      *reinterpret_cast<uint4*>(layers[y].K + to) = *(reinterpret_cast<const uint4*>(t.k + from) + i);
      *reinterpret_cast<uint4*>(layers[y].V + to) = *(reinterpret_cast<const uint4*>(t.v + from) + i);
    }
    return;
  }
  const int rs = fm_ring(l), at = r.b * rs + r.p % rs;
  float *h = l == 0 ? hc_ring : hv_ring, *tri = l == 1 ? triv_ring : trif_ring, *z = l == 0 ? zc : (l == 1 ? zv : zf);
  for (int i = threadIdx.x; i < d; i += blockDim.x) {
    z[(size_t)at * d + i] = t.z[l][(size_t)row * d + i];
    if (l < 2) h[(size_t)at * d + i] = t.h[l][(size_t)row * d + i];
    if (l > 0)
      for (int k = 0; k < 3; ++k) tri[((size_t)at * 3 + k) * d + i] = t.tri[l - 1][((size_t)row * 3 + k) * d + i];
  }
}

}  // namespace ht
