"""Rows of an attention call that belong to no tree, and trees of more nodes than the call allows for: what they get, and what is
recorded.  Tables with room for many positions make a pass of few a large one, which takes the large tiles."""
import numpy as np
import pytest

import test_gpu_tree_ops as T
import tree_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

if torch.cuda.is_available():
    from paper_2511_15618_b200 import FmError

BF = torch.bfloat16
ROOM = {"small": None, "large": 4000}           # pages of 16 in a table


def poisoned(*shapes):
    """The blocks that the next allocations of these sizes will get hold sevens."""
    held = [torch.full(s, 7.0, device="cuda", dtype=d) for s, d in shapes]
    torch.cuda.synchronize()
    del held


def case(room, lens, trees, heads, Hkv, dh, extra, seed):
    rng = np.random.default_rng(seed)
    torch.manual_seed(seed)
    c = T.filled(rng, lens, Hkv, dh, 16, BF, max_pages=ROOM[room])
    rows = sum(map(len, trees)) + extra
    q, kn, vn = (torch.randn((rows, h, dh), device="cuda").to(BF) for h in (heads, Hkv, Hkv))
    return c, q, kn, vn


def agree(c, lens, trees, heads, got, q, kn, vn, at, most):
    """Row ranges `at` of the trees against the plain form of their first `most` nodes."""
    for b, (n, tree, r0) in enumerate(zip(lens, trees, at)):
        m = min(len(tree), most)
        if m == 0:
            continue
        rows = slice(r0, r0 + m)
        k, v = T.gathered(c, 0, b, n, kn[rows], vn[rows])
        want, wl, to, tl = R.attention(q[rows].double().cpu().numpy(), k, v, R.visible(tree[:m], n, 0, 0), c.head_dim ** -0.5, T.UNIT[BF])
        assert (np.abs(got[0][rows].double().cpu().numpy() - want) <= to).all()
        live = ~np.isneginf(wl)
        assert (np.abs(got[1][rows].double().cpu().numpy() - wl)[live] <= tl[live]).all()


@pytest.mark.parametrize("room", ["small", "large"])
@pytest.mark.parametrize("dh,heads,Hkv", [(64, 2, 2), (128, 4, 1)])
@pytest.mark.parametrize("nodes,most", [(300, None), (300, 256), (40, 7), (5, 1), (257, None)])
def test_a_tree_of_more_nodes_than_there_is_room_for(room, dh, heads, Hkv, nodes, most):
    rng = np.random.default_rng(nodes)
    lens, trees = [70, 33, 5], [T.random_tree(rng, n) for n in (1, nodes, 3)]
    c, q, kn, vn = case(room, lens, trees, heads, Hkv, dh, 0, nodes)
    off = np.concatenate([[0], np.cumsum([len(t) for t in trees])])
    poisoned((q.shape, BF), (q.shape[:2], torch.float32))
    got = c.attention(0, q, kn, vn, T.dev(off), T.dev(sum(trees, [])), max_nodes=most, want_lse=True)
    room_for = most or 256
    agree(c, lens, trees, heads, got, q, kn, vn, off, room_for)
    for b, tree in enumerate(trees):
        rows = slice(off[b] + min(len(tree), room_for), off[b + 1])
        assert (got[0][rows] == 0).all() and torch.isneginf(got[1][rows]).all()
    with pytest.raises(FmError) as e:
        c.check()
    assert e.value.code == -3
    c.check()
    kept = torch.full(q.shape, 7.0, device="cuda", dtype=BF)
    c.attention(0, q, kn, vn, T.dev(off), T.dev(sum(trees, [])), max_nodes=most, out=kept)
    for b, tree in enumerate(trees):
        rows = slice(off[b], off[b] + min(len(tree), room_for))
        assert torch.equal(kept[rows], got[0][rows]) and (kept[rows.stop:off[b + 1]] == 7).all()


@pytest.mark.parametrize("room", ["small", "large"])
@pytest.mark.parametrize("before,behind", [(0, 1), (3, 0), (2, 500)])
def test_rows_in_front_of_and_behind_the_trees(room, before, behind):
    lens, trees = [70, 33], [[-1, 0, 0], [-1, 0]]
    c, q, kn, vn = case(room, lens, trees, 4, 2, 64, before + behind, 3)
    off = np.array([0, 3, 5]) + before
    parent = T.dev([5] * before + sum(trees, []) + [5] * behind)
    poisoned((q.shape, BF), (q.shape[:2], torch.float32))
    got = c.attention(0, q, kn, vn, T.dev(off), parent, want_lse=True)
    c.check()
    agree(c, lens, trees, 4, got, q, kn, vn, off, 256)
    for rows in (slice(0, before), slice(before + 5, None)):
        assert (got[0][rows] == 0).all() and torch.isneginf(got[1][rows]).all()
    kept = torch.full(q.shape, 7.0, device="cuda", dtype=BF)
    poisoned((q.shape[:2], torch.float32))
    _, lse = c.attention(0, q, kn, vn, T.dev(off), parent, want_lse=True, out=kept)
    assert (kept[:before] == 7).all() and (kept[before + 5:] == 7).all() and torch.equal(lse, got[1])


@pytest.mark.parametrize("room", ["small", "large"])
def test_a_captured_call_of_a_padded_batch(room):
    """A graph for eight rows, replayed with fewer of them in use."""
    lens = [70, 33]
    c, q, kn, vn = case(room, lens, [[-1] * 4, [-1] * 4], 2, 2, 64, 0, 4)
    off, parent = T.dev([0, 4, 8]), T.dev([-1, 0, 1, 2] * 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.default_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            held = c.attention(0, q, kn, vn, off, parent, want_lse=True)
    for used in ([0, 4, 8], [0, 1, 2], [0, 0, 3], [2, 2, 2]):
        off.copy_(T.dev(used))
        held[0].fill_(7.0), held[1].fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        out, lse = c.attention(0, q, kn, vn, off, parent, want_lse=True)
        assert torch.equal(held[0], out) and torch.equal(held[1], lse)
        rest = [r for r in range(8) if not used[0] <= r < used[2]]
        assert (out[rest] == 0).all() and torch.isneginf(lse[rest]).all()
        given = [-1, 0, 1, 2] * 2                                        # (a tree that starts inside these: parents that are no earlier nodes)
        agree(c, lens, [given[used[0]:used[1]], given[used[1]:used[2]]], 2, (out, lse), q, kn, vn, used, 256)
    c.check()
