"""Calls on trees and pages that have nothing to do: no rows, no trees, no entries."""
import pytest

import test_gpu_tree_ops as T

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF = torch.bfloat16


def cache():
    c = T.PagedCache(2, 8, 4, 2, 64, 3, 4)
    c.reserve(T.dev([0, 1]), T.dev([3, 4]))
    rows = torch.randn((2, 3, 2, 64), device="cuda").to(BF)
    c.append(T.dev([0]), rows, rows, T.dev([0, 3]))
    return c


def none(*shape, dtype=BF):
    return torch.empty(shape, device="cuda", dtype=dtype)


@pytest.mark.parametrize("trees", [0, 1, 3])
def test_attention_of_no_rows(trees):
    c = cache()
    off, parent = T.dev([0] * (trees + 1)), none(0, dtype=torch.int32)
    out, lse = c.attention(1, none(0, 4, 64), none(0, 2, 64), none(0, 2, 64), off, parent, want_lse=True)
    assert out.shape == (0, 4, 64) and out.dtype == BF and lse.shape == (0, 4)
    given = none(0, 4, 64)
    assert c.attention(1, none(0, 4, 64), none(0, 2, 64), none(0, 2, 64), off, parent, out=given).data_ptr() == given.data_ptr()
    c.check()


@pytest.mark.parametrize("trees", [0, 1, 5])
def test_acceptance_of_no_rows(trees):
    empty = none(0, dtype=torch.int32)
    path, n_acc, nxt = T.tree_accept(empty, empty, T.dev([0] * (trees + 1)), empty, max_nodes=4)
    assert path.tolist() == [[-1] * 4] * trees and n_acc.tolist() == [0] * trees and nxt.tolist() == [-1] * trees
    if trees:                                              # rows that are not there
        _, n_acc, nxt = T.tree_accept(empty, empty, T.dev([0] * trees + [3]), empty)
        assert n_acc.tolist() == [0] * trees and nxt.tolist() == [-1] * trees


@pytest.mark.parametrize("paths", [False, True])
def test_appends_of_no_rows(paths):
    c = cache()
    before = [t.clone() for t in (c.k, c.v, c.table, c.lens, c.refs)]
    kw = dict(path=T.dev([[-1, -1]] * 2), n_acc=T.dev([0, 0])) if paths else {}
    c.append(T.dev([0, 1]), none(2, 0, 2, 64), none(2, 0, 2, 64), T.dev([0, 0, 0]), **kw)
    c.check()
    c.append(T.dev([0, 1]), none(2, 0, 2, 64), none(2, 0, 2, 64), T.dev([0, 0, 0]), max_rows=5, **kw)
    c.check()
    # rows that are not there
    kw = dict(path=T.dev([[0, 1]] * 2), n_acc=T.dev([2, 0])) if paths else {}
    c.append(T.dev([0, 1]), none(2, 0, 2, 64), none(2, 0, 2, 64), T.dev([0, 2, 2]), max_rows=5, **kw)
    with pytest.raises(T.FmError) as e:
        c.check()
    assert e.value.code == -1
    for empty in (c.fork, c.reserve, c.truncate):
        empty(none(0, dtype=torch.int32), none(0, dtype=torch.int32))
    c.append(none(0, dtype=torch.int32), none(2, 0, 2, 64), none(2, 0, 2, 64), T.dev([0]))
    c.check()
    assert all(torch.equal(a, b) for a, b in zip(before, (c.k, c.v, c.table, c.lens, c.refs)))
