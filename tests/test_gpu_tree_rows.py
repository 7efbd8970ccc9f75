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
        assert (np.abs(got[1][rows].double().cpu().numpy()[live] - wl[live]) <= tl[live]).all()


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


BAD = [[0, 3, 9], [0, 3, 2 ** 31 - 1], [0, -4, 8], [-1, 3, 8], [5, 3, 8], [-2 ** 31, 2 ** 31 - 1, -2 ** 31], [8, 8, 9], [2 ** 31 - 1, 3, 8], [3, -2 ** 31, 8]]


def fits(off, i, rows=8):
    return 0 <= off[i] <= off[i + 1] <= rows


@pytest.mark.parametrize("room", ["small", "large"])
@pytest.mark.parametrize("off", BAD)
def test_offsets_that_are_not_inside_the_rows(room, off):
    """Eight rows; a tree whose rows are not among them is one without rows, the other one is what it is alone."""
    lens = [70, 33]
    c, q, kn, vn = case(room, lens, [[-1] * 4, [-1] * 4], 2, 2, 64, 0, 5)
    parent = [-1, 0, 1, 2, -1, -1, 5, 0]
    poisoned((q.shape, BF), (q.shape[:2], torch.float32))
    got = c.attention(0, q, kn, vn, T.dev(off), T.dev(parent), want_lse=True)
    with pytest.raises(FmError) as e:
        c.check()
    assert e.value.code == -1
    trees = [parent[off[i]:off[i + 1]] if fits(off, i) else [] for i in range(2)]
    agree(c, lens, trees, 2, got, q, kn, vn, off, 256)
    rest = [r for r in range(8) if not any(fits(off, i) and off[i] <= r < off[i + 1] for i in range(2))]
    assert (got[0][rest] == 0).all() and torch.isneginf(got[1][rest]).all()


@pytest.mark.parametrize("off", BAD)
@pytest.mark.parametrize("paths", [False, True])
def test_appended_offsets_that_are_not_inside_the_rows(off, paths):
    c = T.PagedCache(2, 20, 4, 1, 64, 2, 10)
    kn, vn = (torch.randn((2, 8, 1, 64), device="cuda").to(BF) for _ in range(2))
    c.reserve(T.dev([0, 1]), T.dev([8, 8]))
    kw = dict(path=T.dev([[0], [0]]), n_acc=T.dev([1, 1])) if paths else {}
    c.append(T.dev([0, 1]), kn, vn, T.dev(off), **kw)
    took = [off[i + 1] - off[i] if fits(off, i) else 0 for i in range(2)]
    took = [min(n, 1) for n in took] if paths else took
    assert c.lens.tolist() == took
    for i, n in enumerate(took):
        for j in range(n):
            assert torch.equal(c.k[:, c.table[i, j // 4].long(), :, j % 4], kn[:, off[i] + j])
    # (offsets that descend inside the rows are those of an entry without rows; with a path it names rows that are not its own)
    if paths or any(off[i] < 0 or off[i + 1] > 8 for i in range(2)):
        with pytest.raises(FmError) as e:
            c.check()
        assert e.value.code == -1
    else:
        c.check()


@pytest.mark.parametrize("off", BAD)
def test_accepted_offsets_that_are_not_inside_the_rows(off):
    tokens, parent, predicted = [1, 2, 3, 4, 1, 2, 3, 4], [-1, 0, 1, 2, -1, -1, 5, 0], [2, 3, 4, 5, 2, 3, 4, 5]
    path, n_acc, nxt = T.tree_accept(T.dev(tokens), T.dev(parent), T.dev(off), T.dev(predicted))
    for i in range(2):
        at = slice(off[i], off[i + 1]) if fits(off, i) else slice(0, 0)
        want, behind = R.accept(tokens[at], parent[at], predicted[at])
        assert n_acc[i].item() == len(want) and nxt[i].item() == behind and path[i].tolist() == want + [-1] * (8 - len(want))


@pytest.mark.parametrize("room", ["small", "large"])
@pytest.mark.parametrize("dh,heads,Hkv", [(64, 4, 2), (128, 8, 1)])
def test_outputs_in_the_place_of_the_queries(room, dh, heads, Hkv):
    rng = np.random.default_rng(9)
    lens, trees = [1500, 3, 260], [T.random_tree(rng, n) for n in (60, 1, 33)]
    c, q, kn, vn = case(room, lens, trees, heads, Hkv, dh, 0, 9)
    off, parent = T.dev(np.concatenate([[0], np.cumsum([len(t) for t in trees])])), T.dev(sum(trees, []))
    want, lse = c.attention(0, q, kn, vn, off, parent, want_lse=True)
    got, again = c.attention(0, q, kn, vn, off, parent, want_lse=True, out=q)
    assert got.data_ptr() == q.data_ptr() and torch.equal(got, want) and torch.equal(again, lse)
