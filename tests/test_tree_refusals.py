"""What the calls on trees, pages and scores refuse, on the host and without a device: an error return comes before anything is
enqueued.  And the plain definitions that the device tests compare with, on cases worked out by hand."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import tree_reference as R

from paper_2511_15618_b200 import trees as T
from paper_2511_15618_b200.build import build

INVALID, CAPACITY, UNSUPPORTED = -1, -3, -6
P = 1 << 20                                    # an address that nothing dereferences, 256-byte aligned


@pytest.fixture(scope="module")
def lib():
    build()
    return T._lib()


def cache(**kw):
    c = T.FmCache(P, P, 0, 64 * 16 * 2, 64 * 16, 64, 2, 10, 16, 2, 64, T.FM_BF16)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def pages(**kw):
    p = T.FmPages(10, 16, 4, 5, P, P, P, P, P)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def args(**kw):
    a = T.FmTreeArgs(P, P, P, P, None, 256, 128, 256, P, P, None, P, P, None, 5, 4, 2, 4, 8, 80, 0, 0, 0.125)
    for k, v in kw.items():
        setattr(a, k, v)
    return bytes(a)


def refused(call, *args, **kw):
    with pytest.raises(T.FmError) as e:
        call(*args, **kw)
    return e.value.code == INVALID


def test_tensors_without_a_device_are_refused(lib):
    """The functions for torch tensors: what is no tensor, of another type or shape, or on the host."""
    torch = pytest.importorskip("torch")
    x, i = torch.zeros(3, 5), torch.zeros(3, dtype=torch.int32)
    for logits in (x, x[0], x.double(), x[:, :0], None, 3):
        assert refused(T.logprobs, logits)
    assert refused(T.tree_accept, i, i, i, i) and refused(T.tree_accept, i, None, i, i) and refused(T.tree_accept, i[None], i, i, i)
    host = T._host()
    c, p = cache(), pages()
    at = C.addressof(c), C.addressof(p), 0
    q, kv = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    good = [0, q, kv, kv, i[:2], i, None, 0, 0, None, None, None, False, None]
    for k, bad in ((0, None), (0, 1 << 40), (1, None), (1, q[0]), (1, q.float()), (2, q), (3, None), (4, i[:0]), (7, 2.5), (9, "x"), (13, x), (1, q)):
        a = list(good)
        a[k] = bad
        assert refused(host.attention, *at, *a), (k, bad)
    assert refused(host.attention, *at) and refused(host.attention, 0, *at[1:], *good)
    rows = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    for a in ([i, rows, rows, i], [i[:2], rows, rows, i, None, i], [i[:2], rows[0], rows, i], [i[:2], rows, rows, i]):
        assert refused(host.append, *at, *(a + [None] * (7 - len(a))))


def test_work_sizes(lib):
    assert lib.fm_pages_work_ints(10, 4) > 0
    for n, s in ((0, 4), (10, 0), (-1, 4), (10, T.FM_MAX_SEQS + 1)):
        assert lib.fm_pages_work_ints(n, s) == 0


@pytest.mark.parametrize("bad", [dict(table=None), dict(lens=None), dict(refs=None), dict(status=None), dict(work=None), dict(n_pages=0),
                                 dict(page_slots=0), dict(max_seqs=0), dict(max_seqs=5000), dict(max_pages=0)])
def test_pages_refuse(lib, bad):
    p, c = pages(**bad), cache()
    rows = bytes(T.FmNewRows(P, P, 0, 128, 64))
    assert lib.fm_pages_reset(p, None) == INVALID
    assert lib.fm_pages_fork(p, P, P, 1, None) == INVALID
    assert lib.fm_pages_truncate(p, P, P, 1, None) == INVALID
    assert lib.fm_pages_reserve(p, c, P, P, 1, None) == INVALID
    assert lib.fm_pages_append(p, c, rows, P, P, None, 0, None, 1, 1, None) == INVALID
    assert lib.fm_pages_compact(p, c, None, None) == INVALID


def test_page_lists_refuse(lib):
    p, c, rows = pages(), cache(), T.FmNewRows(P, P, 0, 128, 64)
    for call in (lambda a, b, n: lib.fm_pages_fork(p, a, b, n, None), lambda a, b, n: lib.fm_pages_truncate(p, a, b, n, None),
                 lambda a, b, n: lib.fm_pages_reserve(p, c, a, b, n, None)):
        assert call(None, P, 1) == INVALID and call(P, None, 1) == INVALID and call(P, P, -1) == INVALID
        assert call(P, P, T.FM_MAX_SEQS + 1) == CAPACITY and call(None, None, 0) == 0
    assert lib.fm_pages_reserve(p, c, P, P, 5, None) == INVALID          # more entries than sequences
    append = lambda rows=rows, path=None, stride=0, acc=None, n=1, most=1: lib.fm_pages_append(p, c, bytes(rows), P, P, path, stride, acc, n, most, None)
    assert append(n=0) == 0
    for kw in (dict(path=P), dict(path=P, stride=4), dict(path=P, acc=P), dict(most=-1), dict(n=5), dict(rows=T.FmNewRows(None, P, 0, 128, 64)),
               dict(rows=T.FmNewRows(P + 8, P, 0, 128, 64)), dict(rows=T.FmNewRows(P, P, 4, 128, 64)), dict(rows=T.FmNewRows(P, P, 0, 127, 64)),
               dict(rows=T.FmNewRows(P, P, 0, 128, 63))):
        assert append(**kw) == INVALID, kw


@pytest.mark.parametrize("bad,code", [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=P + 2), INVALID), (dict(n_layers=0), INVALID),
                                      (dict(n_pages=9), INVALID), (dict(page_slots=8), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=0), INVALID),
                                      (dict(head_dim=60), INVALID), (dict(slot_stride=63), INVALID), (dict(head_stride=4), INVALID),
                                      (dict(page_stride=12), INVALID), (dict(layer_stride=2), INVALID), (dict(dtype=T.FM_FP32), UNSUPPORTED),
                                      (dict(n_layers=40000), CAPACITY)])
def test_caches_refuse(lib, bad, code):
    p, c = pages(), cache(**bad)
    assert lib.fm_pages_reserve(p, c, P, P, 1, None) == code
    assert lib.fm_pages_compact(p, c, None, None) == code


def test_a_table_of_too_many_positions(lib):
    assert lib.fm_pages_reset(pages(max_pages=1 << 27), None) == CAPACITY
    assert lib.fm_tree_attention_bytes(cache(), args(max_pages=1 << 27)) == 0


@pytest.mark.parametrize("bad,code", [(dict(q=None), INVALID), (dict(k_new=None), INVALID), (dict(v_new=None), INVALID), (dict(out=None), INVALID),
                                      (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(row_off=None), INVALID), (dict(parent=None), INVALID),
                                      (dict(q=P + 4), INVALID), (dict(out=P + 8), INVALID), (dict(batch=0), INVALID), (dict(n_heads=0), INVALID),
                                      (dict(n_heads=3), INVALID), (dict(max_nodes=0), INVALID), (dict(max_len=-1), INVALID), (dict(window=-1), INVALID),
                                      (dict(n_prefix=-1), INVALID), (dict(max_pages=0), INVALID), (dict(max_seqs=0), INVALID),
                                      (dict(q_row_stride=252), INVALID), (dict(q_row_stride=248), INVALID), (dict(new_row_stride=120), INVALID),
                                      (dict(out_row_stride=248), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
                                      (dict(batch=T.FM_MAX_TREES + 1), CAPACITY), (dict(max_nodes=T.FM_MAX_TREE_NODES + 1), CAPACITY)])
def test_attention_refuses(lib, bad, code):
    assert lib.fm_tree_attention_bytes(cache(), args()) > 0
    assert lib.fm_tree_attention_bytes(cache(), args(**bad)) == 0
    assert lib.fm_tree_attention(cache(), 0, args(**bad), P, 1 << 30, None) == code


def test_attention_refuses_heads_layers_and_workspaces(lib):
    size = lib.fm_tree_attention_bytes(cache(), args())
    assert lib.fm_tree_attention(cache(head_dim=32), 0, args(), P, size, None) == UNSUPPORTED
    assert lib.fm_tree_attention(cache(head_dim=96, n_kv_heads=1), 0, args(q_row_stride=512, out_row_stride=512), P, size, None) == UNSUPPORTED
    assert lib.fm_tree_attention(cache(dtype=T.FM_FP32), 0, args(), P, size, None) == UNSUPPORTED
    assert lib.fm_tree_attention(cache(), -1, args(), P, size, None) == INVALID
    assert lib.fm_tree_attention(cache(), 2, args(), P, size, None) == INVALID
    assert lib.fm_tree_attention(cache(), 0, args(), None, size, None) == INVALID
    assert lib.fm_tree_attention(cache(), 0, args(), P + 16, size, None) == INVALID
    assert lib.fm_tree_attention(cache(), 0, args(), P, size - 1, None) == CAPACITY


def test_accept_refuses(lib):
    good = [P, P, P, P, 2, P, 4, P, P]
    for i, bad in [(0, None), (1, None), (2, None), (3, None), (4, 0), (5, None), (6, 0), (7, None), (8, None)]:
        a = list(good)
        a[i] = bad
        assert lib.fm_tree_accept(*a, None) == INVALID, i


def test_scores_refuse(lib):
    good = dict(x=P, dtype=T.FM_FP32, rows=2, vocab=50, stride=50, top=3)
    def call(**kw):
        g = {**good, **kw}
        return lib.fm_logprobs(g["x"], g["dtype"], g["rows"], g["vocab"], g["stride"], P, P, P, P, g["top"], P, P, None)
    for bad in (dict(x=None), dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(stride=49), dict(top=-1), dict(top=51), dict(x=P + 2),
                dict(x=P + 1, dtype=T.FM_BF16)):
        assert call(**bad) == INVALID, bad
    assert call(top=33) == CAPACITY
    assert call(rows=0) == 0


def test_division_of_slots_by_the_page_size():
    """The multiplication that the kernels divide with, from the source's formula: exact for every slot below 2^31."""
    text = open(os.path.join(os.path.dirname(T.__file__), "csrc", "fm_ops.cu")).read()
    body = re.search(r"Div div_by\(int d\) \{(.*?)\n\}", text, re.S).group(1)
    assert "const int p = 31 + l;" in body and "((1ull << p) + d - 1) / d" in body and "v.shift = p - 32" in body and "(1ll << l) < d" in body
    rng = np.random.default_rng(0)
    for d in list(range(2, 300)) + [1000, 4095, 4096, 4097, 65535, 2 ** 20 + 1, 2 ** 30 - 1, 2 ** 30]:
        l = (d - 1).bit_length()
        mul, shift = -(-(1 << (31 + l)) // d), l - 1
        assert mul < 2 ** 32
        n = np.concatenate([rng.integers(0, 2 ** 31, 500), [0, 1, d - 1, d, d + 1, 2 ** 31 - 1], np.arange(1, 200) * d % 2 ** 31, (np.arange(1, 200) * d - 1) % 2 ** 31])
        for x in n.tolist():
            assert (x * mul >> 32) >> shift == x // d


# ---------------------------------------------------------------------------- the plain definitions
def test_ancestors_and_what_a_node_sees():
    assert R.ancestors([-1, 0, 1, 0, -2, 4, 7, -1]) == [{0}, {0, 1}, {0, 1, 2}, {0, 3}, set(), set(), set(), {7}]
    see = R.visible([-1, 0, 0], 4, 3, 1)
    # window 3, one conditioning slot: the root (position 4) sees 0, 2, 3 and itself; its children 0, 3, the root, themselves
    assert see.astype(int).tolist() == [[1, 0, 1, 1, 1, 0, 0], [1, 0, 0, 1, 1, 1, 0], [1, 0, 0, 1, 1, 0, 1]]


def test_attention_of_one_key_and_of_two():
    q, k, v = np.ones((1, 1, 2)), np.array([[[0.0, 0.0], [np.log(3.0), 0.0]]]), np.array([[[1.0, 0.0], [5.0, 4.0]]])
    out, lse, _, _ = R.attention(q, k, v, np.array([[True, True]]), 1.0, 0.0)
    assert np.allclose(out[0, 0], [4.0, 3.0]) and np.isclose(lse[0, 0], np.log(4.0))
    out, lse, _, _ = R.attention(q, k, v, np.array([[True, False]]), 1.0, 0.0)
    assert np.allclose(out[0, 0], [1.0, 0.0]) and lse[0, 0] == 0.0


def test_accepted_path_takes_the_lowest_child():
    assert R.accept([9, 4, 4, 5], [-1, 0, 0, 1], [4, 5, 7, 8]) == ([0, 1, 3], 8)
    assert R.accept([9, 3, 4, 5], [-1, 0, 0, 2], [4, 5, 7, 8]) == ([0, 2], 7)
    assert R.accept([9, 3], [-2, 0], [3, 3]) == ([], -1)


def test_pages_of_lists():
    data = {(0, 0): np.arange(5 * 2, dtype=float).reshape(5, 1, 2, 1)}
    p = R.Pages(5, 2, 3, 4, data)
    p.reserve([1, 0], [3, 1])
    assert p.table() == [[2, -1, -1, -1], [0, 1, -1, -1], [-1] * 4]
    rows = {(0, 0): np.array([[[70.0]], [[71.0]], [[72.0]], [[80.0]]])}
    p.append([1, 0], [0, 3, 4], rows)
    p.fork([1], [2])
    assert p.refs() == [2, 2, 1, 0, 0]
    p.reserve([2, 1], [1, 1])                                            # the copy goes first, the source keeps its page
    assert p.tables == [[2], [0, 1], [0, 3]] and data[(0, 0)][3, 0, 0, 0] == 72.0
    p.truncate([1, 0], [0, 0])
    assert p.refs() == [1, 0, 0, 1, 0] and p.compact() == 2 and p.tables[2] == [0, 1] and data[(0, 0)][1, 0, 0, 0] == 72.0


def test_pages_too_large_to_count(lib):
    p, c = pages(page_slots=1 << 27, max_pages=1), cache(page_slots=1 << 27, n_kv_heads=2, head_dim=64)
    assert lib.fm_pages_compact(p, c, None, None) == CAPACITY                # 2^27 slots x 2 heads x 8 pieces
    assert lib.fm_tree_attention_bytes(c, args(max_pages=1)) == 0
