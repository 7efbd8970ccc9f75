"""Softmax weights far below the row's largest: a sink that takes nearly all of the weight and whose values are nothing, and a tail
that makes the output; scores that rise along the cache.  Tables with room for many positions take the large tiles."""
import numpy as np
import pytest

import test_gpu_tree_ops as T
import tree_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF, HF = torch.bfloat16, torch.float16
ROOM = {"small": None, "large": 4000}           # pages of 16 in a table


def pool(room, lens, Hkv, dh, dtype, seed):
    rng = np.random.default_rng(seed)
    torch.manual_seed(seed)
    return T.filled(rng, lens, Hkv, dh, 16, dtype, max_pages=ROOM[room])


def put(c, b, keys, values):
    """keys, values [positions, dh] into all heads of a sequence."""
    at = torch.arange(keys.shape[0], device="cuda")
    page = c.table[b].long()[at // 16]
    c.k[0, page, :, at % 16] = keys[:, None].to(c.dtype)
    c.v[0, page, :, at % 16] = values[:, None].to(c.dtype)


def compare(c, lens, tree, q, kn, vn, got, step):
    """As check_attention, with a weight's rounding half a step of the type or half of `step` of the row's largest, whichever is more."""
    n = len(tree)
    for b, length in enumerate(lens):
        rows = slice(b * n, (b + 1) * n)
        k, v = T.gathered(c, 0, b, length, kn[rows], vn[rows])
        see = R.visible(tree, length, 0, 0)
        Q = q[rows].double().cpu().numpy()
        want, wl, to, tl = R.attention(Q, k, v, see, c.head_dim ** -0.5, T.UNIT[c.dtype])
        for h in range(Q.shape[1]):
            hk = h // (Q.shape[1] // k.shape[0])
            for i in range(n):
                at = np.nonzero(see[i])[0]
                largest = np.exp((c.head_dim ** -0.5 * (k[hk][at] @ Q[i, h])).max() - wl[i, h])
                to[i, h] += step / 2 * largest * np.abs(v[hk][at]).sum(0)
        out, lse = got[0][rows].double().cpu().numpy(), got[1][rows].double().cpu().numpy()
        # (the output itself: half has no number below 2^-24, so it is off by half of that at most)
        assert (np.abs(out - want) <= to + 2.0 ** -25).all(), float((np.abs(out - want) / to).max())
        assert (np.abs(lse - wl) <= tl).all()


@pytest.mark.parametrize("room", ["small", "large"])
@pytest.mark.parametrize("dh,heads", [(64, 1), (64, 40), (128, 1), (128, 40)])
@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("below", [10.0, 15.3, 21.3, 26.0, 30.0])
def test_a_tail_below_the_sinks(room, dh, heads, dtype, below):
    """Every sixteenth key is a sink, so every slice of a chunk has one; the others lie 2^below under it and carry the values."""
    lens, tree = [1500, 700], [-1, 0]
    c = pool(room, lens, 1, dh, dtype, int(below))
    for b, n in enumerate(lens):
        keys, values = torch.zeros((n, dh), device="cuda"), torch.rand((n, dh), device="cuda") * 3e4 + 2e4
        keys[::16, 0] = below / 1.4426950408889634 * dh ** 0.5 / 8
        values[::16] = 0
        put(c, b, keys, values)
    q = torch.zeros((4, heads, dh), device="cuda", dtype=dtype)
    q[:, :, 0] = 8
    kn, vn = (torch.zeros((4, 1, dh), device="cuda", dtype=dtype) for _ in range(2))
    kn[:, :, 0] = -4                                                      # the nodes lie below the tail
    got = c.attention(0, q, kn, vn, T.dev([0, 2, 4]), T.dev(tree * 2), want_lse=True)
    compare(c, lens, tree, q, kn, vn, got, 2.0 ** -33 if dtype is HF else 0.0)


@pytest.mark.parametrize("room", ["small", "large"])
@pytest.mark.parametrize("dh,heads", [(64, 2), (64, 40), (128, 2), (128, 40)])
@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("bits", [-90.0, -7.0, 3.0, 4.9, 5.1, 9.0, 20.0, 90.0])
def test_scores_that_rise_or_fall_along_the_cache(room, dh, heads, dtype, bits):
    """By so many powers of two a chunk of 128, in all rows or, half of them, half as fast: the reference of the exponentials moves or stays."""
    lens, tree = [1300, 400], [-1, 0]
    c = pool(room, lens, 1, dh, dtype, int(bits) + 100)
    for b, n in enumerate(lens):
        keys, values = torch.zeros((n, dh), device="cuda"), torch.randn((n, dh), device="cuda")
        keys[:, 0] = torch.arange(n, device="cuda") // 16 / 8 * bits / 1.4426950408889634 * dh ** 0.5 / 8
        put(c, b, keys, values)
    q = torch.zeros((4, heads, dh), device="cuda", dtype=dtype)
    q[:, 0::2, 0], q[:, 1::2, 0] = 8, 4
    kn, vn = (torch.randn((4, 1, dh), device="cuda").to(dtype) for _ in range(2))
    got = c.attention(0, q, kn, vn, T.dev([0, 2, 4]), T.dev(tree * 2), want_lse=True)
    compare(c, lens, tree, q, kn, vn, got, 2.0 ** -33 if dtype is HF else 0.0)
