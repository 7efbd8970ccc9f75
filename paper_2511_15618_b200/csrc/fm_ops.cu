// C ABI of the calls that need no context: trees of drafts over a paged cache, token scores (see include/flashmesh.h).
// The host checks the arguments, picks a kernel by sizes and types and enqueues it.
#include "../../include/flashmesh.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <numeric>

#include "fm_logprobs.cuh"
#include "fm_pages.cuh"
#include "fm_tree.cuh"

namespace {

constexpr int64_t MOST_SLOTS = 1 << 30;      // positions a table can hold
constexpr int MOST_GRID = 65535;
constexpr int MOST_PIECES = 1 << 30;         // 16-byte pieces of a page, or of the rows that an entry appends: counted in 32 bits

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline cudaStream_t as_stream(void* s) { return reinterpret_cast<cudaStream_t>(s); }
inline int launched() { return cudaGetLastError() == cudaSuccess ? FM_OK : FM_ERR_CUDA; }

// The kernel's blocks may start while those of the one in front still run: all of them wait for its end first (griddepcontrol.wait)
template <typename Kernel, typename... Args>
int launch(Kernel kern, dim3 grid, int block, int smem, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, args...) == cudaSuccess ? FM_OK : FM_ERR_CUDA;
}

// the kernel may use that much shared memory on the current device (asked once per device)
template <typename Kernel>
bool allow_smem(Kernel kern, int bytes, std::atomic<uint64_t>& asked) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return false;
  if (dev < 64 && ((asked.load() >> dev) & 1)) return true;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  if (dev < 64) asked.fetch_or(1ull << dev);
  return true;
}

int check_pages(const fm_pages* p) {
  if (p == nullptr || p->table == nullptr || p->lens == nullptr || p->refs == nullptr || p->status == nullptr || p->work == nullptr) return FM_ERR_INVALID_ARG;
  if (p->page_slots < 1 || p->max_pages < 1 || fm_pages_work_ints(p->n_pages, p->max_seqs) == 0) return FM_ERR_INVALID_ARG;
  if ((int64_t)p->max_pages * p->page_slots > MOST_SLOTS) return FM_ERR_CAPACITY;
  return FM_OK;
}

int check_cache(const fm_cache* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || !aligned16(c->k) || !aligned16(c->v)) return FM_ERR_INVALID_ARG;
  if (c->n_layers < 1 || c->n_pages < 1 || c->page_slots < 1 || c->n_kv_heads < 1) return FM_ERR_INVALID_ARG;
  if ((c->layer_stride | c->page_stride | c->head_stride | c->slot_stride) & 7) return FM_ERR_INVALID_ARG;
  if (c->head_dim < 8 || c->head_dim % 8 != 0) return FM_ERR_INVALID_ARG;
  if (c->dtype != FM_BF16 && c->dtype != FM_FP16) return FM_ERR_UNSUPPORTED;
  if (c->n_layers > MOST_GRID / 2 - 1) return FM_ERR_CAPACITY;
  if ((int64_t)c->page_slots * c->n_kv_heads * (c->head_dim / 8) > MOST_PIECES) return FM_ERR_CAPACITY;
  return FM_OK;
}

int check_both(const fm_pages* p, const fm_cache* c) {
  int rc = check_pages(p);
  if (rc == FM_OK) rc = check_cache(c);
  if (rc == FM_OK && (p->n_pages != c->n_pages || p->page_slots != c->page_slots)) rc = FM_ERR_INVALID_ARG;
  return rc;
}

int check_list(const int32_t* a, const int32_t* b, int32_t n) {
  if (n < 0 || (n > 0 && (a == nullptr || b == nullptr))) return FM_ERR_INVALID_ARG;
  return n > FM_MAX_SEQS ? FM_ERR_CAPACITY : FM_OK;
}

pg::Geo geo_of(const fm_cache& c) {
  pg::Geo g;
  g.k = static_cast<char*>(c.k); g.v = static_cast<char*>(c.v);
  g.layer = 2 * c.layer_stride; g.page = 2 * c.page_stride; g.head = 2 * c.head_stride; g.slot = 2 * c.slot_stride;
  g.layers = c.n_layers; g.heads = c.n_kv_heads; g.row16 = c.head_dim / 8;
  return g;
}

int check_tree(const fm_cache* c, const fm_tree_args* t) {
  const int rc = check_cache(c);
  if (rc != FM_OK) return rc;
  if (t == nullptr || t->q == nullptr || t->k_new == nullptr || t->v_new == nullptr || t->out == nullptr || t->table == nullptr || t->lens == nullptr ||
      t->row_off == nullptr || t->parent == nullptr) return FM_ERR_INVALID_ARG;
  if (!aligned16(t->q) || !aligned16(t->k_new) || !aligned16(t->v_new) || !aligned16(t->out)) return FM_ERR_INVALID_ARG;
  if (t->batch < 1 || t->n_heads < 1 || t->n_heads % c->n_kv_heads != 0 || t->max_nodes < 1 || t->max_len < 0 || t->window < 0 || t->n_prefix < 0 ||
      t->max_pages < 1 || t->max_seqs < 1) return FM_ERR_INVALID_ARG;
  if ((t->q_row_stride | t->new_row_stride | t->out_row_stride) & 7) return FM_ERR_INVALID_ARG;
  if (t->q_row_stride < (int64_t)t->n_heads * c->head_dim || t->out_row_stride < (int64_t)t->n_heads * c->head_dim ||
      t->new_row_stride < (int64_t)c->n_kv_heads * c->head_dim) return FM_ERR_INVALID_ARG;
  if (t->n_rows < 0 || (t->fill & ~(FM_FILL_OUT | FM_FILL_LSE)) != 0 || (t->fill != 0 && t->n_rows == 0)) return FM_ERR_INVALID_ARG;
  if (!(t->scale > 0.f) || t->scale - t->scale != 0.f) return FM_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FM_ERR_UNSUPPORTED;
  if (t->batch > FM_MAX_TREES || t->max_nodes > FM_MAX_TREE_NODES || (int64_t)t->max_pages * c->page_slots > MOST_SLOTS) return FM_ERR_CAPACITY;
  return FM_OK;
}

template <typename T, int R>
int score_short(const lp::Args& a, cudaStream_t stream) {
  return launch(lp::short_kernel<T, R>, dim3(a.rows / lp::SHORT_WARPS + (a.rows % lp::SHORT_WARPS != 0)), 32 * lp::SHORT_WARPS, 0, stream, a);
}

// Rows whose vectors fit into a warp's registers (64 values a lane) take a warp, longer ones a block: of 256 threads, or of 512
// where there are too few rows to fill the SMs with the smaller one.
template <typename T>
int score_rows(const lp::Args& a, cudaStream_t stream) {
  constexpr int N = lp::Vec<T>::N, MOST = 64 / N;
  const int vectors = (a.vocab / N + 31) / 32;               // a lane
  if (vectors <= MOST) {
    if (vectors <= 1) return score_short<T, 1>(a, stream);
    if (vectors <= MOST / 4) return score_short<T, MOST / 4>(a, stream);
    if (vectors <= MOST / 2) return score_short<T, MOST / 2>(a, stream);
    return score_short<T, MOST>(a, stream);
  }
  if (a.rows >= 2 * 148) return launch(lp::long_kernel<T, 256, 8>, dim3(a.rows), 256, 8 * 256 * 16, stream, a);
  static std::atomic<uint64_t> asked{0};
  if (!allow_smem(lp::long_kernel<T, 512, 8>, 8 * 512 * 16, asked)) return FM_ERR_CUDA;
  return launch(lp::long_kernel<T, 512, 8>, dim3(a.rows), 512, 8 * 512 * 16, stream, a);
}

// The form of a pass, by what the caller says of its sizes (bounds that are far above them take the other form: right, and
// slower: 64 single tokens over 4000 positions each, called without bounds, 245 us for 176).  Rows that share keys (nodes x heads of a group): up to 16 take tiles of
// 16 rows, warp-level products (a batch of 64, one node, 8 kv-heads of 128, 4000 positions: 176 us).  More rows would each have
// the keys brought again, from L2 at best, so they take tensor-core tiles of 256 - but those start and end slower, and a tile
// of 256 is one CTA's: passes too small to fill the SMs take the small tiles too.  Measured where a CTA has so many chunks
// (OVER more a tile), small | large tiles: 2 tiles of 16, 12 chunks 23 | 41 us, 51 chunks 55 | 55, 112 chunks 97 | 78;
// 4 to 16 tiles, 7 chunks 21 | 35 us, 15 chunks 25 | 51 and 23 | 23, 22 chunks 31 | 35 and 37 | 33, 36 chunks 41 | 38.
inline bool few_rows(const tr::Args& a, int head_dim) {
  const int64_t rows = (int64_t)a.max_nodes * a.G, tiles = (rows + 15) / 16;
  if (tiles == 1) return true;
  const int chunk = head_dim == 64 ? tr::Rows16<64>::C : tr::Rows16<128>::C;
  const int64_t seen = a.window > 0 ? std::min<int64_t>(a.max_len, (int64_t)a.n_prefix + a.window) : a.max_len;
  const int64_t chunks = (seen + chunk - 1) / chunk + (a.max_nodes + chunk - 1) / chunk + tr::OVER;
  return a.batch * a.Hkv * tiles * chunks <= (tiles == 2 ? 64 : 24) * tr::SMS;
}
using tr::DESC_BYTES;
static_assert(DESC_BYTES >= tr::SMS * sizeof(int4), "");
static_assert(tr::Rows16<64>::C == 128 && tr::Rows256<64>::C == 128 && tr::Rows256<128>::C == 128 && tr::Rows16<128>::C == 64, "make_maps");
static_assert(tr::Rows16<128>::FIXED + tr::plan_bytes(FM_MAX_TREES) <= 227 * 1024 && tr::Rows256<128>::FIXED + tr::plan_bytes(FM_MAX_TREES) <= 227 * 1024, "");

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
  }();
  return fn;
}
// A layer's pool as (features, slots, heads, pages), boxes of 64 features and the most slots that divide pages and chunks evenly,
// 128-byte swizzle (a function of the address: a box may start at any row of 128 bytes).  Page sizes that take more boxes than a
// warp has lanes, and strides that a map cannot hold, are copied by threads.  (One page a sequence: a chunk's slots, what lies
// behind the last one reads as zeros.)
bool make_maps_of(const fm_cache& c, int layer, int max_pages, int chunk, tr::Args& a) {
  const int ps = c.page_slots;
  a.box_rows = max_pages == 1 && ps >= chunk ? chunk : std::gcd(ps, chunk);
  if (a.box_rows * 32 < chunk) return false;                 // (a lane each)
  const EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const int64_t most = (int64_t)1 << 39;
  for (int64_t s : {c.slot_stride, c.head_stride, c.page_stride})
    if (s <= 0 || s >= most) return false;
  const cuuint64_t dim[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)ps, (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  const cuuint64_t stride[3] = {(cuuint64_t)c.slot_stride * 2, (cuuint64_t)c.head_stride * 2, (cuuint64_t)c.page_stride * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)a.box_rows, 1, 1}, one[4] = {1, 1, 1, 1};
  const CUtensorMapDataType type = c.dtype == FM_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  for (int kv = 0; kv < 2; ++kv) {
    char* base = static_cast<char*>(kv == 0 ? c.k : c.v) + 2 * layer * c.layer_stride;
    if (fn(kv == 0 ? &a.map_k : &a.map_v, type, 4, base, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return false;
  }
  return true;
}

// Will no tile be cut, whatever the lengths?  (See tr::make_plan: at most a tile per CTA, of eight chunks at most.)
inline bool whole_for_sure(const tr::Args& a, int rows, int chunk, int ctas) {
  const int64_t tiles = (int64_t)a.batch * a.Hkv * (((int64_t)a.max_nodes * a.G + rows - 1) / rows);
  return tiles <= ctas && (a.max_len + chunk - 1) / chunk + 1 + (a.max_nodes + chunk - 1) / chunk <= 8;
}

template <typename T, int DH>
int tree_attention(const tr::Args& a, cudaStream_t stream) {
  int rc;
  if (few_rows(a, DH)) {
    static std::atomic<uint64_t> asked{0};
    using CF = tr::Rows16<DH>;
    if (!allow_smem(tr::rows16_kernel<T, DH>, CF::bytes(FM_MAX_TREES), asked)) return FM_ERR_CUDA;
    rc = ::launch(tr::rows16_kernel<T, DH>, dim3(tr::SMS), CF::THREADS, CF::bytes(a.batch), stream, a);
    if (rc == FM_OK && !whole_for_sure(a, 16, CF::C, tr::SMS)) rc = ::launch(tr::merge_kernel<T, DH, 16>, dim3(tr::SMS, 4), 256, 0, stream, a);
  } else {
    static std::atomic<uint64_t> asked{0};
    using CF = tr::Rows256<DH>;
    if (!allow_smem(tr::rows256_kernel<T, DH>, CF::bytes(FM_MAX_TREES), asked)) return FM_ERR_CUDA;
    rc = ::launch(tr::rows256_kernel<T, DH>, dim3(tr::SMS), CF::THREADS, CF::bytes(a.batch), stream, a);
    if (rc == FM_OK && !whole_for_sure(a, 256, CF::C, tr::SMS)) rc = ::launch(tr::merge_kernel<T, DH, 256>, dim3(tr::SMS, 16), 256, 0, stream, a);
  }
  return rc;
}

}  // namespace

namespace tr {

Div div_by(int d) {
  Div v{0, 0, d};
  if (d > 1) {
    int l = 0;
    while ((1ll << l) < d) ++l;
    const int p = 31 + l;                      // n * (2^p / d rounded up) >> p is exact for n < 2^31
    v.mul = (uint32_t)(((1ull << p) + d - 1) / d);
    v.shift = p - 32;
  }
  return v;
}
size_t workspace_bytes(int max_nodes, int group, int head_dim) {             // (of more than 16 rows: enough for either form)
  return DESC_BYTES + (size_t)SMS * 2 * ((int64_t)max_nodes * group <= 16 ? 16 : 256) * (head_dim + 2) * sizeof(float);
}
bool make_maps(const fm_cache& c, int layer, int max_pages, Args& a) {
  return make_maps_of(c, layer, max_pages, few_rows(a, c.head_dim) && c.head_dim == 128 ? tr::Rows16<128>::C : 128, a);
}
int launches(const Args& a, int head_dim) {
  const bool few = few_rows(a, head_dim);
  return whole_for_sure(a, few ? 16 : 256, few && head_dim == 128 ? Rows16<128>::C : 128, SMS) ? 1 : 2;
}
int launch(const Args& a, int dtype, int head_dim, cudaStream_t stream) {
  if (dtype == FM_BF16) return head_dim == 64 ? tree_attention<bf16, 64>(a, stream) : tree_attention<bf16, 128>(a, stream);
  return head_dim == 64 ? tree_attention<__half, 64>(a, stream) : tree_attention<__half, 128>(a, stream);
}

}  // namespace tr

extern "C" {

size_t fm_pages_work_ints(int32_t n_pages, int32_t max_seqs) {
  if (n_pages < 1 || max_seqs < 1 || max_seqs > FM_MAX_SEQS) return 0;
  fm_pages p{};
  p.n_pages = n_pages; p.max_seqs = max_seqs;
  return (size_t)pg::word_at(p) + 1;
}

int fm_pages_reset(const fm_pages* p, void* stream) {
  const int rc = check_pages(p);
  if (rc != FM_OK) return rc;
  pg::reset_kernel<<<148, 256, 0, as_stream(stream)>>>(*p);
  return launched();
}

int fm_pages_fork(const fm_pages* p, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  int rc = check_pages(p);
  if (rc == FM_OK) rc = check_list(src, dst, n);
  if (rc != FM_OK || n == 0) return rc;
  return launch(pg::fork_kernel, dim3(n), 128, 0, as_stream(stream), *p, src, dst, (int)n);
}

int fm_pages_reserve(const fm_pages* p, const fm_cache* c, const int32_t* seqs, const int32_t* grow, int32_t n, void* stream) {
  int rc = check_both(p, c);
  if (rc == FM_OK) rc = check_list(seqs, grow, n);
  if (rc == FM_OK && n > p->max_seqs) rc = FM_ERR_INVALID_ARG;       // (the jobs of the entries have a place each)
  if (rc != FM_OK || n == 0) return rc;
  rc = launch(pg::reserve_plan_kernel, dim3(1), pg::PLAN, 0, as_stream(stream), *p, seqs, grow, (int)n);
  return rc != FM_OK ? rc : launch(pg::reserve_copy_kernel, dim3(n, 2 * c->n_layers), 256, 0, as_stream(stream), *p, geo_of(*c));
}

int fm_pages_append(const fm_pages* p, const fm_cache* c, const fm_new_rows* rows, const int32_t* seqs, const int32_t* row_off, const int32_t* path,
                    int32_t path_stride, const int32_t* n_acc, int32_t n, int32_t max_rows, void* stream) {
  int rc = check_both(p, c);
  if (rc == FM_OK) rc = check_list(seqs, row_off, n);
  if (rc == FM_OK && n > p->max_seqs) rc = FM_ERR_INVALID_ARG;
  if (rc != FM_OK) return rc;
  if (rows == nullptr || rows->k == nullptr || rows->v == nullptr || !aligned16(rows->k) || !aligned16(rows->v) || max_rows < 0 || rows->n_rows < 0)
    return FM_ERR_INVALID_ARG;
  if ((rows->layer_stride | rows->row_stride | rows->head_stride) & 7) return FM_ERR_INVALID_ARG;
  if (path != nullptr && (n_acc == nullptr || path_stride < 1)) return FM_ERR_INVALID_ARG;
  if (n == 0) return FM_OK;
  pg::Rows r;
  r.k = static_cast<const char*>(rows->k); r.v = static_cast<const char*>(rows->v);
  r.layer = 2 * rows->layer_stride; r.row = 2 * rows->row_stride; r.head = 2 * rows->head_stride;
  r.n_rows = rows->n_rows;
  const int most = 2 * c->n_layers, share = (148 * 3 + n - 1) / n;           // blocks of an entry: a wave over all entries at most
  return launch(pg::append_kernel, dim3(n, share < most ? share : most), 256, 0, as_stream(stream), *p, geo_of(*c), r, seqs, row_off, path, (int)path_stride, n_acc,
                std::min<int>(max_rows, MOST_PIECES / (c->n_kv_heads * (c->head_dim / 8))));
}

int fm_pages_truncate(const fm_pages* p, const int32_t* seqs, const int32_t* new_lens, int32_t n, void* stream) {
  int rc = check_pages(p);
  if (rc == FM_OK) rc = check_list(seqs, new_lens, n);
  if (rc != FM_OK || n == 0) return rc;
  return launch(pg::truncate_kernel, dim3(n), 128, 0, as_stream(stream), *p, seqs, new_lens);
}

int fm_pages_compact(const fm_pages* p, const fm_cache* c, int32_t* used, void* stream) {
  int rc = check_both(p, c);
  if (rc == FM_OK) rc = launch(pg::compact_plan_kernel, dim3(1), pg::PLAN, 0, as_stream(stream), *p, used);
  if (rc != FM_OK) return rc;
  // enough blocks for every SM; no more than there can be pages to move
  const int rows = 2 * c->n_layers + 1, most = p->n_pages / 2 + 1, want = (148 * 16 + rows - 1) / rows;
  return launch(pg::compact_copy_kernel, dim3(want < most ? want : most, rows), 256, 0, as_stream(stream), *p, geo_of(*c));
}

size_t fm_tree_attention_bytes(const fm_cache* cache, const fm_tree_args* args) {
  if (check_tree(cache, args) != FM_OK) return 0;
  return tr::workspace_bytes(args->max_nodes, args->n_heads / cache->n_kv_heads, cache->head_dim);
}

int fm_tree_attention(const fm_cache* c, int32_t layer, const fm_tree_args* t, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_tree(c, t);
  if (rc != FM_OK) return rc;
  if (layer < 0 || layer >= c->n_layers || workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return FM_ERR_INVALID_ARG;
  if (workspace_bytes < fm_tree_attention_bytes(c, t)) return FM_ERR_CAPACITY;
  tr::Args a{};
  a.q = t->q; a.k_new = t->k_new; a.v_new = t->v_new; a.out = t->out; a.lse = t->lse;
  a.q_row = t->q_row_stride; a.new_row = t->new_row_stride; a.out_row = t->out_row_stride;
  a.k = static_cast<const char*>(c->k) + 2 * layer * c->layer_stride;
  a.v = static_cast<const char*>(c->v) + 2 * layer * c->layer_stride;
  a.page = c->page_stride; a.head = c->head_stride; a.slot = c->slot_stride;
  a.table = t->table; a.lens = t->lens; a.seqs = t->seqs; a.row_off = t->row_off; a.parent = t->parent; a.status = t->status;
  a.desc = static_cast<int4*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + DESC_BYTES);
  a.page_div = tr::div_by(c->page_slots); a.g_div = tr::div_by(t->n_heads / c->n_kv_heads);
  a.n_pages = c->n_pages; a.max_pages = t->max_pages; a.max_seqs = t->max_seqs; a.batch = t->batch;
  a.H = t->n_heads; a.Hkv = c->n_kv_heads; a.G = t->n_heads / c->n_kv_heads; a.max_nodes = t->max_nodes;
  const int64_t holds = (int64_t)t->max_pages * c->page_slots;
  a.max_len = t->max_len < holds ? t->max_len : (int)holds;
  a.window = t->window; a.n_prefix = t->n_prefix;
  a.n_rows = t->n_rows; a.fill = t->fill;
  a.scale_log2 = t->scale * 1.4426950408889634f;
  a.tma = tr::make_maps(*c, layer, t->max_pages, a) ? 1 : 0;
  return tr::launch(a, c->dtype, c->head_dim, as_stream(stream));
}

int fm_tree_accept(const int32_t* tokens, const int32_t* parent, const int32_t* row_off, const int32_t* predicted, int32_t batch, int32_t* path,
                   int32_t path_stride, int32_t* n_acc, int32_t* next_tok, void* stream) {
  return fm_tree_accept_rows(tokens, parent, row_off, predicted, INT32_MAX, batch, path, path_stride, n_acc, next_tok, stream);
}

int fm_tree_accept_rows(const int32_t* tokens, const int32_t* parent, const int32_t* row_off, const int32_t* predicted, int32_t rows, int32_t batch,
                        int32_t* path, int32_t path_stride, int32_t* n_acc, int32_t* next_tok, void* stream) {
  if (tokens == nullptr || parent == nullptr || row_off == nullptr || predicted == nullptr || path == nullptr || n_acc == nullptr || next_tok == nullptr)
    return FM_ERR_INVALID_ARG;
  if (rows < 0 || batch < 1 || path_stride < 1) return FM_ERR_INVALID_ARG;
  return launch(tr::accept_kernel, dim3(batch / 4 + (batch % 4 != 0)), 128, 0, as_stream(stream), tokens, parent, row_off, predicted, (int)batch, (int)rows, path,
                (int)path_stride, n_acc, next_tok);
}

int fm_logprobs(const void* logits, int32_t dtype, int32_t rows, int32_t vocab, int64_t row_stride, const int32_t* tokens, float* logprob, float* entropy,
                int32_t* rank, int32_t top, int32_t* top_ids, float* top_logprobs, void* stream) {
  if (logits == nullptr || rows < 0 || vocab < 1 || row_stride < vocab || top < 0 || top > vocab) return FM_ERR_INVALID_ARG;
  if (dtype != FM_BF16 && dtype != FM_FP16 && dtype != FM_FP32) return FM_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(logits) & (dtype == FM_FP32 ? 3 : 1)) != 0) return FM_ERR_INVALID_ARG;
  if (top > FM_MAX_TOP) return FM_ERR_CAPACITY;
  if (rows == 0) return FM_OK;
  lp::Args a{logits, tokens, logprob, entropy, rank, top_ids, top_logprobs, row_stride, rows, vocab, top_ids == nullptr && top_logprobs == nullptr ? 0 : top};
  if (dtype == FM_FP32) return score_rows<float>(a, as_stream(stream));
  if (dtype == FM_BF16) return score_rows<bf16>(a, as_stream(stream));
  return score_rows<__half>(a, as_stream(stream));
}

}  // extern "C"
