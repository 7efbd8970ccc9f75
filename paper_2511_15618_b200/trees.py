"""Trees of drafts over a paged cache, and token scores: binding of the calls of include/flashmesh.h that need no context.

`PagedCache` owns (or is laid over) the tensors of a pool of cache pages and forwards to the C entry points, by way of native
functions that check the tensors (csrc/trees_host.cpp); `tree_accept` and `logprobs` are functions of tensors.  Everything is
enqueued on torch's current stream of the tensors' device, allocates through torch and can be captured into a CUDA graph.
There is no CPU path, and no backward pass: an input that requires a gradient is refused where gradients are recorded.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding as _b
from .binding import FmError

FM_BF16, FM_FP16, FM_FP32 = 0, 1, 2
FM_MAX_TOP = 32
FM_MAX_TREE_NODES = 256
FM_MAX_SEQS = 4096
FM_MAX_TREES = 512


class FmCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64), ("head_stride", C.c_int64),
                ("slot_stride", C.c_int64), ("n_layers", C.c_int32), ("n_pages", C.c_int32), ("page_slots", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class FmPages(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_slots", C.c_int32), ("max_seqs", C.c_int32), ("max_pages", C.c_int32), ("table", C.c_void_p),
                ("lens", C.c_void_p), ("refs", C.c_void_p), ("status", C.c_void_p), ("work", C.c_void_p)]


class FmNewRows(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("row_stride", C.c_int64), ("head_stride", C.c_int64), ("n_rows", C.c_int32)]


class FmTreeArgs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("q_row_stride", C.c_int64), ("new_row_stride", C.c_int64), ("out_row_stride", C.c_int64), ("table", C.c_void_p),
                ("lens", C.c_void_p), ("seqs", C.c_void_p), ("row_off", C.c_void_p), ("parent", C.c_void_p), ("status", C.c_void_p),
                ("max_pages", C.c_int32), ("max_seqs", C.c_int32), ("batch", C.c_int32), ("n_heads", C.c_int32), ("max_nodes", C.c_int32),
                ("max_len", C.c_int32), ("window", C.c_int32), ("n_prefix", C.c_int32), ("scale", C.c_float),
                ("n_rows", C.c_int32), ("fill", C.c_int32)]


_LIB = _HOST = None


def _lib():
    """The library with the types of these calls declared."""
    global _LIB
    if _LIB is None:
        lib = _b.load_library()
        vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        pages, cache = C.POINTER(FmPages), C.POINTER(FmCache)
        for name, res, args in (
                ("fm_pages_work_ints", C.c_size_t, [i32, i32]),
                ("fm_pages_reset", C.c_int, [pages, vp]),
                ("fm_pages_fork", C.c_int, [pages, vp, vp, i32, vp]),
                ("fm_pages_reserve", C.c_int, [pages, cache, vp, vp, i32, vp]),
                ("fm_pages_append", C.c_int, [pages, cache, C.c_char_p, vp, vp, vp, i32, vp, i32, i32, vp]),
                ("fm_pages_truncate", C.c_int, [pages, vp, vp, i32, vp]),
                ("fm_pages_compact", C.c_int, [pages, cache, vp, vp]),
                ("fm_tree_attention_bytes", C.c_size_t, [cache, C.c_char_p]),
                ("fm_tree_attention", C.c_int, [cache, i32, C.c_char_p, vp, C.c_size_t, vp]),
                ("fm_tree_accept", C.c_int, [vp, vp, vp, vp, i32, vp, i32, vp, vp, vp]),
                ("fm_tree_accept_rows", C.c_int, [vp, vp, vp, vp, i32, i32, vp, i32, vp, vp, vp]),
                ("fm_logprobs", C.c_int, [vp, i32, i32, i32, i64, vp, vp, vp, vp, i32, vp, vp, vp])):
            getattr(lib, name).restype, getattr(lib, name).argtypes = res, args
        _LIB = lib
    return _LIB


def _host():
    """The native functions of csrc/trees_host.cpp: checks, outputs, workspaces and the call in one."""
    global _HOST
    if _HOST is None:
        _lib()                                             # (built and loaded)
        from . import _trees
        _trees.set_error(FmError)
        _HOST = _trees
    return _HOST


def _need(ok, what):
    if not ok:
        raise FmError(-1, what)


def _check(rc, where):
    if rc != 0:
        raise FmError(rc, where)


def _ids(t, device, what):
    """Address of a contiguous int32 vector or matrix on the device."""
    if t.dtype is not torch.int32 or t.device != device or not t.is_contiguous():
        raise FmError(-1, f"{what}: a contiguous int32 tensor on {device}")
    return t.data_ptr()


class PagedCache:
    """Keys and values of `max_seqs` sequences in pages of `page_slots` positions, the same page ids in every layer.

    k, v: [n_layers, n_pages, n_kv_heads, page_slots, head_dim] (bfloat16 or float16); table [max_seqs, max_pages], lens
    [max_seqs], refs [n_pages], status [1]: int32.  `check()` raises what the device has recorded in status.
    Calls on one cache have to be ordered: one stream, or streams that wait for one another."""

    def __init__(self, n_layers, n_pages, page_slots, n_kv_heads, head_dim, max_seqs, max_pages, dtype=None, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("PagedCache needs a CUDA device; there is no CPU path")
        shape = (n_layers, n_pages, n_kv_heads, page_slots, head_dim)
        k, v = (torch.zeros(shape, dtype=dtype or torch.bfloat16, device=device) for _ in range(2))
        i32 = dict(dtype=torch.int32, device=device)
        self._lay(k, v, torch.full((max_seqs, max_pages), -1, **i32), torch.zeros(max_seqs, **i32), torch.zeros(n_pages, **i32))

    @classmethod
    def over(cls, k, v, table, lens, refs):
        """A cache over tensors that exist (strides of k and v are free but for the last; both have the same)."""
        self = cls.__new__(cls)
        self._lay(k, v, table, lens, refs)
        return self

    def _lay(self, k, v, table, lens, refs):
        types = {torch.bfloat16: FM_BF16, torch.float16: FM_FP16}
        _need(k.dim() == 5 and k.is_cuda and k.dtype in types and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device,
              "PagedCache: k and v [layers, pages, kv heads, slots, head_dim] in bfloat16 or float16 on one device")
        _need(not (k.requires_grad or v.requires_grad), "PagedCache: keys and values that require a gradient: there is no backward pass")
        _need(k.stride() == v.stride() and k.stride(4) == 1, "PagedCache: k and v with the same strides, the last 1")
        _need(table.dim() == 2 and lens.shape == table.shape[:1] and refs.shape == k.shape[1:2], "PagedCache: table [seqs, pages], lens [seqs], refs [pool]")
        lib = _lib()
        self.k, self.v, self.table, self.lens, self.refs = k, v, table, lens, refs
        self.device, self.dtype = k.device, k.dtype
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_slots, self.head_dim = k.shape
        self.max_seqs, self.max_pages = table.shape
        ints = lib.fm_pages_work_ints(self.n_pages, self.max_seqs)
        _need(ints > 0, "PagedCache: number of pages or sequences")
        self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.work = torch.zeros(ints, dtype=torch.int32, device=self.device)
        s = k.stride()
        self._cache = FmCache(k.data_ptr(), v.data_ptr(), s[0], s[1], s[2], s[3], self.n_layers, self.n_pages, self.page_slots, self.n_kv_heads,
                              self.head_dim, types[k.dtype])
        self._pages = FmPages(self.n_pages, self.page_slots, self.max_seqs, self.max_pages, _ids(table, self.device, "table"),
                              _ids(lens, self.device, "lens"), _ids(refs, self.device, "refs"), self.status.data_ptr(), self.work.data_ptr())
        self._at = C.addressof(self._cache), C.addressof(self._pages), self.device.index
        self._held = table, lens, refs                     # what the calls write: marked as written in place
        self._all = (k, v) + self._held

    def check(self):
        """Waits for the device; raises FmError for the error it has recorded (of several the lowest code), and clears it."""
        torch.cuda.synchronize(self.device)                # (calls on any of its streams)
        code = int(self.status.item())
        if code != 0:
            self.status.zero_()
            raise FmError(code, "PagedCache")

    def reset(self):
        """All pages free, all sequences empty."""
        with torch.cuda.device(self.device):
            _check(_lib().fm_pages_reset(C.byref(self._pages), torch.cuda.current_stream().cuda_stream), "fm_pages_reset")
        torch.autograd.graph.increment_version(self._held)

    def fork(self, src, dst):
        """Sequences dst become copies of src that share their pages (int32 lists on the device; negative: skipped)."""
        _host().fork(*self._at, src, dst, *self._held)

    def reserve(self, seqs, grow):
        """Pages of their own for grow[i] more positions of sequence seqs[i] (a shared last page is copied)."""
        _host().reserve(*self._at, seqs, grow, *self._all)

    def append(self, seqs, k_new, v_new, row_off, path=None, n_acc=None, max_rows=None):
        """Write rows of k_new, v_new [layers, rows, kv heads, head_dim] behind the sequences and advance their lengths: all rows
        row_off[i]..row_off[i+1]-1 of entry i, or those that path [n, stride] / n_acc [n] name (see `tree_accept`)."""
        _host().append(*self._at, seqs, k_new, v_new, row_off, path, n_acc, max_rows, self.k, self.v, self.lens)

    def truncate(self, seqs, lens):
        """Cut sequences seqs[i] to at most lens[i] positions and give back the pages behind them (0: all)."""
        _host().truncate(*self._at, seqs, lens, *self._held)

    def compact(self):
        """Move the pages in use to the front of the pool; returns their number (int32 [1], on the device)."""
        return _host().compact(*self._at, self.table, *self._all)

    def attention(self, layer, q, k_new, v_new, row_off, parent, seqs=None, window=0, n_prefix=0, scale=None, max_nodes=None, max_len=None,
                  want_lse=False, out=None):
        """Attention of the nodes of trees over the cached positions and their ancestors in one layer.

        q [rows, heads, head_dim], k_new, v_new [rows, kv heads, head_dim] (rows may lie apart); row_off [n + 1]; parent [rows]: an earlier
        node of the tree, counted from its first row, or -1.  seqs [n]: the trees' sequences (None: 0 .. n-1).  max_nodes, max_len:
        bounds on a tree's nodes and a sequence's positions (default: what there is room for).  They choose the kernel too: say them where they are
        known, or single tokens of a batch are taken for one tree of many nodes.  Returns out, or (out, lse).

        A tree of more nodes than max_nodes, or than FM_MAX_TREE_NODES, is recorded for `check`; the nodes behind take no part.  So are offsets that do not
        ascend inside the rows.  Rows of no tree,
        theirs and those in front of the first or behind the last tree, are 0, their lse -inf; an `out` that is given keeps them."""
        return _host().attention(*self._at, layer, q, k_new, v_new, row_off, parent, seqs, window, n_prefix, scale, max_nodes, max_len, want_lse, out)


def tree_accept(tokens, parent, row_off, predicted, max_nodes=None):
    """The longest path of every tree that the predictions confirm: (path [n, max_nodes] node indices, then -1; n_acc [n];
    next_token [n]).  tokens, parent, predicted [rows], row_off [n + 1]: int32 on the device."""
    return _host().accept(tokens, parent, row_off, predicted, max_nodes)


def logprobs(logits, tokens=None, top=0):
    """Scores of logits rows [rows, vocab] (float32, bfloat16 or float16; rows may lie apart): (logprob [rows], entropy [rows], rank
    [rows], top_ids [rows, top], top_logprobs [rows, top]).  tokens: int32 [rows], or None (logprob -inf, rank -1)."""
    return _host().logprobs(logits, tokens, top)
