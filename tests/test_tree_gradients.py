"""The calls on trees, pages and scores have no backward pass: inputs that ask for a gradient are refused, not answered without one
(CPU); what is written in place counts as written (GPU)."""
import ctypes as C

import pytest

import test_tree_refusals as R
from test_tree_refusals import lib                         # noqa: F401 (the built library)

torch = pytest.importorskip("torch")


def refused_for_a_gradient(call, *args):
    with pytest.raises(R.T.FmError) as e:
        call(*args)
    return e.value.code == R.INVALID and "gradient" in str(e.value)


def test_inputs_that_require_a_gradient(lib):              # noqa: F811
    """(Tensors on the host are refused too; the gradient is what is said first.)"""
    i = torch.zeros(3, dtype=torch.int32)
    x = torch.zeros(3, 5, requires_grad=True)
    for logits in (x, x * 2, x.bfloat16()):
        assert refused_for_a_gradient(R.T.logprobs, logits)
        with torch.no_grad():
            assert not refused_for_a_gradient(R.T.logprobs, logits)
        assert not refused_for_a_gradient(R.T.logprobs, logits.detach())
    host = R.T._host()
    c, p = R.cache(), R.pages()
    at = C.addressof(c), C.addressof(p), 0
    q, kv = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    good = [0, q, kv, kv, i[:2], i, None, 0, 0, None, None, None, False, None]
    for k in (1, 2, 3):
        a = list(good)
        a[k] = a[k].clone().requires_grad_()
        assert refused_for_a_gradient(host.attention, *at, *a), k
        with torch.no_grad():
            assert not refused_for_a_gradient(host.attention, *at, *a), k
    rows = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    for a in ([rows.clone().requires_grad_(), rows], [rows, rows.clone().requires_grad_()]):
        assert refused_for_a_gradient(host.append, *at, i[:2], *a, i, None, None, None)


@pytest.mark.gpu
def test_outputs_in_place_and_a_cache_count_as_written():
    from paper_2511_15618_b200 import PagedCache
    c = PagedCache(2, 8, 4, 1, 64, 2, 4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    kn, vn = (torch.randn((2, 3, 1, 64), device="cuda").bfloat16() for _ in range(2))
    tensors = lambda: dict(k=c.k, v=c.v, table=c.table, lens=c.lens, refs=c.refs)

    def changes(call):
        before = {n: (t._version, t.clone()) for n, t in tensors().items()}
        call()
        for n, t in tensors().items():
            version, value = before[n]
            assert torch.equal(t, value) or t._version > version, n      # what changed was marked
    changes(lambda: c.reserve(i32([0, 1]), i32([3, 2])))
    changes(lambda: c.append(i32([0]), kn, vn, i32([0, 3])))
    changes(lambda: c.fork(i32([0]), i32([1])))
    changes(lambda: c.reserve(i32([1]), i32([3])))
    changes(lambda: c.append(i32([1]), kn, vn, i32([0, 2])))
    changes(lambda: c.truncate(i32([0]), i32([0])))
    changes(c.compact)
    changes(c.reset)
    # a gradient whose formula needs what was overwritten is refused by torch
    w = torch.ones(c.k.shape, device="cuda", requires_grad=True)
    y = (w * c.k).sum()
    c.reserve(i32([0]), i32([3]))
    c.append(i32([0]), kn, vn, i32([0, 3]))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    q = torch.randn((3, 1, 64), device="cuda").bfloat16()
    out = torch.zeros_like(q)
    version = out._version
    c.attention(0, q, kn[0], vn[0], i32([0, 3]), i32([-1, 0, 1]), out=out)
    assert out._version > version
    with torch.inference_mode():                           # (tensors without a count)
        inner = torch.zeros_like(q)
        c.attention(0, q, kn[0], vn[0], i32([0, 3]), i32([-1, 0, 1]), out=inner)
        c.truncate(i32([0]), i32([1]))
    assert torch.equal(inner, out)
    w = torch.randn(c.k.shape, device="cuda").bfloat16().requires_grad_()
    with pytest.raises(Exception, match="gradient"):
        PagedCache.over(w, w, c.table, c.lens, c.refs)
