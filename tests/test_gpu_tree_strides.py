"""Tensors with dimensions of size 1, whose strides mean nothing: a transposed or selected view of one head, one row or one layer is
what its contents are."""
import numpy as np
import pytest

import test_gpu_tree_ops as T

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF = torch.bfloat16


def odd(x, *dims):
    """The same contents, with a stride of 3 (no multiple of what copies need) wherever a listed dimension has size 1."""
    assert all(x.shape[d] == 1 for d in dims)
    return x.as_strided(x.shape, [3 if d in dims else s for d, s in enumerate(x.stride())])


@pytest.mark.parametrize("heads,rows", [(1, 5), (4, 1), (1, 1)])
def test_attention_of_one_head_or_one_row(heads, rows):
    rng = np.random.default_rng(rows)
    c = T.filled(rng, [40], 1, 64, 16, BF)
    tree = [-1, 0, 0, 1, 1][:rows]
    q, kn, vn = (torch.randn((rows, h, 64), device="cuda").to(BF) for h in (heads, 1, 1))
    args = T.dev([0, rows]), T.dev(tree)
    want = c.attention(0, q, kn, vn, *args, want_lse=True)
    T.check_attention(c, 0, [40], [tree], heads, got=want, q=q, kn=kn, vn=vn)
    ones = [d for d, n in enumerate((rows, heads)) if n == 1]
    out = odd(torch.zeros_like(q), *ones)
    got = c.attention(0, odd(q, *ones), odd(kn, 1), vn, *args, want_lse=True, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # as a projection gives them: [batch 1, rows, heads, dim] with the heads in front
    view = lambda x: x.unsqueeze(0).transpose(1, 2)[0].transpose(0, 1)
    got = c.attention(0, view(q), view(kn), view(vn), *args, want_lse=True)
    assert torch.equal(got[0], want[0])


@pytest.mark.parametrize("layers,rows,heads", [(1, 3, 2), (2, 1, 2), (2, 3, 1), (1, 1, 1)])
def test_appends_of_one_layer_row_or_head(layers, rows, heads):
    c = T.PagedCache(layers, 8, 4, heads, 64, 2, 4)
    kn, vn = (torch.randn((layers, rows, heads, 64), device="cuda").to(BF) for _ in range(2))
    c.reserve(T.dev([0]), T.dev([rows]))
    ones = [d for d, n in enumerate((layers, rows, heads)) if n == 1]
    c.append(T.dev([0]), odd(kn, *ones), vn, T.dev([0, rows]))
    c.check()
    assert c.lens.tolist() == [rows, 0]
    for pool, new in ((c.k, kn), (c.v, vn)):
        assert torch.equal(pool[:, 0, :, :rows], new.transpose(1, 2))


def test_views_that_differ_are_refused():
    c = T.PagedCache(2, 8, 4, 2, 64, 2, 4)
    kn, vn = (torch.randn((3, 2, 64), device="cuda").to(BF) for _ in range(2))
    q = torch.randn((3, 4, 64), device="cuda").to(BF)
    apart = lambda x: torch.empty_strided(x.shape, (x.stride(0) + 64, 64, 1), device="cuda", dtype=BF).copy_(x)
    turned = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
    args = T.dev([0, 3]), T.dev([-1, 0, 0])
    c.attention(0, q, apart(kn), apart(vn), *args)
    for bad in ((q, apart(kn), vn), (turned(q), kn, vn), (q, turned(kn), turned(vn))):
        with pytest.raises(T.FmError) as e:
            c.attention(0, *bad, *args)
        assert e.value.code == -1
