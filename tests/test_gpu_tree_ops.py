"""Trees of drafts over a paged cache and token scores on the device, against plain definitions in 64 bits."""
import numpy as np
import pytest

import tree_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

if torch.cuda.is_available():
    from paper_2511_15618_b200 import FmError, PagedCache, logprobs, tree_accept

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
BF, HF = torch.bfloat16, torch.float16


def dev(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(device="cuda", dtype=dtype)


def random_tree(rng, n, prune=0.0):
    p = [-1]
    for i in range(1, n):
        p.append(-2 if rng.random() < prune else (-1 if rng.random() < 0.05 else (i - 1 if rng.random() < 0.5 else int(rng.integers(i)))))
    return p[:n]


def filled(rng, lens, Hkv, dh, page, dtype, layers=1, spare=3, max_pages=None, holes=True):
    """A pool whose sequences hold `lens` positions in shuffled pages."""
    have = [-(-n // page) for n in lens]
    n_pages = sum(have) + spare
    order = rng.permutation(n_pages)
    max_pages = max_pages or max(max(have), 1)
    c = PagedCache(layers, n_pages, page, Hkv, dh, len(lens), max_pages, dtype=dtype)
    c.k.copy_(torch.randn(c.k.shape, device="cuda").to(dtype))
    c.v.copy_(torch.randn(c.v.shape, device="cuda").to(dtype))
    table, at = np.full((len(lens), max_pages), -1), 0
    for b, n in enumerate(have):
        table[b, :n] = order[at:at + n]
        at += n
    c.table.copy_(dev(table))
    c.lens.copy_(dev(lens))
    c.refs.copy_(dev(np.bincount(table[table >= 0].astype(int), minlength=n_pages)))
    return c


def gathered(c, layer, b, n, new_k, new_v):
    """[Hkv, n + nodes, dh] float64 keys and values of a sequence and its nodes."""
    out = []
    for pool, new in ((c.k, new_k), (c.v, new_v)):
        pages = c.table[b, :-(-n // c.page_slots)].long()
        old = pool[layer][pages].permute(1, 0, 2, 3).flatten(1, 2)[:, :n]
        out.append(torch.cat([old, new.transpose(0, 1)], 1).double().cpu().numpy())
    return out


def check_attention(c, layer, lens, trees, heads, window=0, prefix=0, scale=None, got=None, q=None, kn=None, vn=None):
    scale = c.head_dim ** -0.5 if scale is None else scale
    out, lse = got
    r = 0
    for b, (n, tree) in enumerate(zip(lens, trees)):
        rows = slice(r, r + len(tree))
        r += len(tree)
        if not tree:
            continue
        k, v = gathered(c, layer, b, n, kn[rows], vn[rows])
        see = R.visible(tree, n, window, prefix)
        v = np.where(see.any(0)[None, :, None], v, 0.0)
        want, wl, to, tl = R.attention(q[rows].double().cpu().numpy(), k, v, see, scale, UNIT[c.dtype])
        o, l = out[rows].double().cpu().numpy(), lse[rows].double().cpu().numpy()
        assert (np.abs(o - want) <= to).all(), (b, float(np.abs(o - want).max()))
        dead = ~see.any(1)                                               # (their lse is -inf on both sides)
        assert (o[dead] == 0).all() and np.isneginf(l[dead]).all()
        assert (np.abs(l[~dead] - wl[~dead]) <= tl[~dead]).all(), b


def run_case(seed, lens, nodes, heads, Hkv, dh, page, dtype, window=0, prefix=0, prune=0.05, scale=None, layers=1, layer=0, **kw):
    rng = np.random.default_rng(seed)
    torch.manual_seed(seed)
    c = filled(rng, lens, Hkv, dh, page, dtype, layers=layers)
    trees = [random_tree(rng, n, prune) for n in nodes]
    rows = sum(nodes)
    q = torch.randn((rows, heads, dh), device="cuda").mul(1.5).to(dtype)
    kn, vn = (torch.randn((rows, Hkv, dh), device="cuda").to(dtype) for _ in range(2))
    off = dev(np.concatenate([[0], np.cumsum(nodes)]))
    got = c.attention(layer, q, kn, vn, off, dev(sum(trees, [])), window=window, n_prefix=prefix, scale=scale, max_nodes=max(nodes), want_lse=True, **kw)
    c.check()
    check_attention(c, layer, lens, trees, heads, window, prefix, scale, got, q, kn, vn)
    return c, trees, q, kn, vn, off, got


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads,Hkv", [(2, 2), (4, 1), (7, 1), (24, 3)])
def test_types_and_heads(dtype, dh, heads, Hkv):
    run_case(1, [37, 0, 200, 1], [5, 3, 9, 1], heads, Hkv, dh, 16, dtype)


@pytest.mark.parametrize("length", [0, 1, 2, 63, 64, 65, 127, 128, 129, 500, 1023, 4100])
@pytest.mark.parametrize("nodes", [1, 4, 28])
def test_lengths(length, nodes):
    run_case(2, [length], [nodes], 4, 2, 64, 64, BF)
    run_case(3, [length, 77], [nodes, 2], 4, 4, 128, 24, HF)


@pytest.mark.parametrize("page", [1, 3, 7, 16, 100, 256])
def test_page_sizes(page):
    run_case(4, [211, 90], [6, 11], 4, 2, 64, page, BF)


@pytest.mark.parametrize("nodes", [2, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 200, 256])
def test_tree_sizes(nodes):
    run_case(5, [70], [nodes], 2, 1, 64, 16, BF)
    run_case(6, [33, 130], [nodes, 1], 8, 1, 128, 16, BF)


@pytest.mark.parametrize("window", [1, 2, 5, 64, 100, 250, 1000])
@pytest.mark.parametrize("prefix", [0, 1, 64, 130, 400])
def test_windows(window, prefix):
    run_case(7, [300, 129, 10], [20, 7, 1], 4, 2, 64, 16, BF, window=window, prefix=prefix)
    run_case(8, [300], [40], 4, 1, 128, 32, HF, window=window, prefix=prefix)


def test_a_long_chain_deeper_than_the_window():
    rng = np.random.default_rng(3)
    c = filled(rng, [50], 1, 64, 16, BF)
    tree = list(range(-1, 255))
    q, kn, vn = (torch.randn((256, 1, 64), device="cuda").to(BF) for _ in range(3))
    got = c.attention(0, q, kn, vn, dev([0, 256]), dev(tree), window=40, n_prefix=3, want_lse=True)
    check_attention(c, 0, [50], [tree], 1, 40, 3, None, got, q, kn, vn)


@pytest.mark.parametrize("batch,heads,Hkv,dh,longest", [(1, 16, 16, 64, 9000), (3, 8, 2, 128, 5000), (40, 4, 4, 64, 700), (200, 2, 1, 64, 300)])
def test_ragged_batches_are_cut_in_any_place(batch, heads, Hkv, dh, longest):
    rng = np.random.default_rng(batch)
    lens = np.exp(rng.uniform(0, np.log(longest), batch)).astype(int).tolist()
    lens[batch // 2] = longest
    nodes = rng.integers(0, 6, batch)
    nodes[0] = 1
    run_case(9, lens, nodes.tolist(), heads, Hkv, dh, 16, BF)


def test_other_layers_sequences_and_scales():
    run_case(10, [100, 40], [4, 4], 2, 2, 64, 16, BF, layers=3, layer=2, scale=0.31)
    rng = np.random.default_rng(11)
    c = filled(rng, [100, 40, 7], 2, 64, 16, BF)
    q = torch.randn((4, 2, 64), device="cuda").to(BF)
    kn, vn = (torch.randn((4, 2, 64), device="cuda").to(BF) for _ in range(2))
    got = c.attention(0, q, kn, vn, dev([0, 2, 3, 4]), dev([-1, 0, -1, -1]), seqs=dev([2, 0, -1]), want_lse=True)
    for rows, b, n in ((slice(0, 2), 2, 7), (slice(2, 3), 0, 100), (slice(3, 4), 0, 0)):
        k, v = gathered(c, 0, b, n, kn[rows], vn[rows])
        tree = [-1, 0] if rows.start == 0 else [-1]
        want, wl, to, tl = R.attention(q[rows].double().cpu().numpy(), k, v, R.visible(tree, n, 0, 0), 64 ** -0.5, UNIT[BF])
        assert (np.abs(got[0][rows].double().cpu().numpy() - want) <= to).all()
        assert (np.abs(got[1][rows].double().cpu().numpy() - wl) <= tl).all()


def test_strides_and_rows_behind_the_last_sequence():
    rng = np.random.default_rng(12)
    lens, nodes, dh = [90, 33], [5, 3], 64
    base = filled(rng, lens, 2, dh, 16, BF)
    # the same pool with slots of all heads side by side: [layer, page, slot, head, dim]
    k, v = (x.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4) for x in (base.k, base.v))
    c = PagedCache.over(k, v, base.table, base.lens, base.refs)
    trees = [random_tree(rng, n) for n in nodes]
    wide = torch.randn((10, 8 * dh), device="cuda").to(BF)                # q | k | v of a fused projection, two rows more than nodes
    q, kn, vn = (wide[:, a * dh:b * dh].unflatten(1, (b - a, dh)) for a, b in ((0, 4), (4, 6), (6, 8)))
    out = torch.full((10, 4 * dh + 64), 7.0, device="cuda", dtype=BF)
    off, parent = dev([0, 5, 8]), dev(sum(trees, []) + [-1, 0])
    got = c.attention(0, q, kn, vn, off, parent, want_lse=True, out=out[:, :4 * dh].unflatten(1, (4, dh)))
    check_attention(c, 0, lens, trees, 4, got=got, q=q, kn=kn, vn=vn)
    assert (out[8:] == 7).all() and (out[:, 4 * dh:] == 7).all()
    again = base.attention(0, q.contiguous(), kn.contiguous(), vn.contiguous(), off, parent, want_lse=True)
    assert torch.equal(again[0][:8], got[0][:8]) and torch.equal(again[1][:8], got[1][:8])


@pytest.mark.parametrize("dh,heads,Hkv,nodes", [(64, 2, 2, 6), (128, 2, 1, 6), (64, 8, 1, 40), (128, 8, 1, 40)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_has_no_effect(dh, heads, Hkv, nodes, what):
    """Values that are not finite in unused pages, behind the length, outside the window, in pruned nodes and in siblings."""
    rng = np.random.default_rng(13)
    lens, window = [150], 60
    c = filled(rng, lens, Hkv, dh, 16, BF)
    tree = [-1, 0, 0, -2] + [1 + i % 2 if i < 2 else (i % 4 + 4 if i > 5 else 4) for i in range(nodes - 4)]
    tree = tree[:nodes]
    q, kn, vn = (torch.randn((nodes, h, dh), device="cuda").to(BF) for h in (heads, Hkv, Hkv))
    clean = c.attention(0, q, kn, vn, dev([0, nodes]), dev(tree), window=window, n_prefix=2, want_lse=True)
    check_attention(c, 0, lens, [tree], heads, window, 2, None, clean, q, kn, vn)
    free = (c.refs == 0).nonzero()[:, 0]
    for x in (c.k, c.v):
        x[:, free] = what
        x[0, c.table[0, 9].long(), :, 150 - 144:] = what
        for s in range(2, 150 - window + 1):
            x[0, c.table[0, s // 16].long(), :, s % 16] = what
    kn[3], vn[3] = what, what                                            # the pruned node
    got = c.attention(0, q, kn, vn, dev([0, nodes]), dev(tree), window=window, n_prefix=2, want_lse=True)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])
    vn[2, :, 5] = what                                                   # a sibling: seen by itself and what lies below it alone
    got = c.attention(0, q, kn, vn, dev([0, nodes]), dev(tree), window=window, n_prefix=2, want_lse=True)
    sees = torch.tensor([2 in a for a in R.ancestors(tree)], device="cuda")
    assert torch.equal(got[0][~sees], clean[0][~sees]) and torch.equal(got[1], clean[1])
    assert not torch.isfinite(got[0][sees][:, :, 5]).any() and torch.isfinite(got[0][sees][:, :, 6:]).all()
    # the oldest position in the root's window, hidden from deeper nodes
    vn[2, :, 5] = 0.0
    s = 150 - window + 1
    c.v[0, c.table[0, s // 16].long(), :, s % 16, 1] = what
    got = c.attention(0, q, kn, vn, dev([0, nodes]), dev(tree), window=window, n_prefix=2, want_lse=True)
    root = torch.tensor([p == -1 for p in tree], device="cuda")
    assert not torch.isfinite(got[0][root][:, :, 1]).any() and torch.isfinite(got[0][~root]).all()


def test_bad_pages_are_refused_on_the_device():
    rng = np.random.default_rng(14)
    c = filled(rng, [40], 1, 64, 16, BF)
    q, kn, vn = (torch.randn((1, 1, 64), device="cuda").to(BF) for _ in range(3))
    for bad in (-1, c.n_pages, 2 ** 30):
        c.table[0, 1] = bad
        out = c.attention(0, q, kn, vn, dev([0, 1]), dev([-1]))
        assert torch.isfinite(out).all()
        with pytest.raises(FmError) as e:
            c.check()
        assert e.value.code == -1
        c.check()


def test_the_same_call_gives_the_same_bits_and_replays():
    c, trees, q, kn, vn, off, got = run_case(15, [3000, 100, 900], [28, 5, 1], 8, 8, 64, 64, BF, window=2000, prefix=64)
    parent = dev(sum(trees, []))
    args = (0, q, kn, vn, off, parent)
    kw = dict(window=2000, n_prefix=64, max_nodes=28, want_lse=True)
    for _ in range(3):
        again = c.attention(*args, **kw)
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.default_stream())
        with torch.cuda.graph(g, stream=side):
            held = c.attention(*args, **kw)
    c.lens[0] = 2500                                                     # lengths are read at every replay
    g.replay()
    torch.cuda.synchronize()
    now = c.attention(*args, **kw)
    assert torch.equal(held[0], now[0]) and not torch.equal(now[0], got[0])


def test_positions_behind_32_bits_of_elements():
    """A pool of more than 2^31 elements: the last pages are found where they are."""
    page, dh, Hkv = 64, 128, 8
    n_pages = 2 ** 31 // (page * dh * Hkv) + 40
    c = PagedCache(1, n_pages, page, Hkv, dh, 1, 4, dtype=BF)
    last = [n_pages - 1, n_pages - 3, 5]
    for p in last:
        c.k[0, p], c.v[0, p] = torch.randn((2, Hkv, page, dh), device="cuda").to(BF)
    c.table[0, :3] = dev(last)
    c.lens[0] = 150
    q = torch.randn((3, 16, dh), device="cuda").to(BF)
    kn, vn = (torch.randn((3, Hkv, dh), device="cuda").to(BF) for _ in range(2))
    got = c.attention(0, q, kn, vn, dev([0, 3]), dev([-1, 0, 0]), want_lse=True)
    check_attention(c, 0, [150], [[-1, 0, 0]], 16, got=got, q=q, kn=kn, vn=vn)


# ------------------------------------------------------------------------------------------ acceptance
@pytest.mark.parametrize("nodes", [1, 2, 10, 33, 100, 256])
def test_accepted_paths(nodes):
    rng = np.random.default_rng(nodes)
    trees, tokens, predicted, off = [], [], [], [0]
    for b in range(37):
        n = nodes if b % 5 else int(rng.integers(0, nodes + 1))
        t = random_tree(rng, n, 0.02)
        if b == 3 and n:
            t[0] = -2
        tok = rng.integers(3, size=n).tolist()
        pre = rng.integers(3, size=n).tolist()
        for i, p in enumerate(t):
            if p >= 0 and rng.random() < 0.7:
                pre[p] = tok[i]
        trees.append(t); tokens.append(tok); predicted.append(pre); off.append(off[-1] + n)
    flat = lambda x: dev(sum(x, []) or [0])
    path, n_acc, nxt = tree_accept(flat(tokens), flat(trees), dev(off), flat(predicted), max_nodes=nodes)
    for b in range(37):
        want, behind = R.accept(tokens[b], trees[b], predicted[b])
        assert n_acc[b].item() == len(want) and nxt[b].item() == behind
        assert path[b].tolist() == want + [-1] * (nodes - len(want))


# ------------------------------------------------------------------------------------------ pages
def host_copy(c):
    data = {(l, kv): pool[l].float().cpu().numpy() for l in range(c.n_layers) for kv, pool in enumerate((c.k, c.v))}
    return R.Pages(c.n_pages, c.page_slots, c.max_seqs, c.max_pages, data)


def same(c, r):
    torch.cuda.synchronize()
    assert c.table.tolist() == r.table()
    assert c.lens.tolist() == r.lens
    assert c.refs.tolist() == r.refs()
    assert c.status.item() == r.status
    for (l, kv), x in r.data.items():
        assert np.array_equal((c.k, c.v)[kv][l].float().cpu().numpy(), x), (l, kv)


@pytest.mark.parametrize("page,Hkv,dh,layers,dtype", [(4, 2, 64, 3, BF), (16, 1, 128, 2, HF), (1, 3, 64, 1, BF), (5, 2, 72, 2, BF)])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_random_histories_of_a_pool(page, Hkv, dh, layers, dtype, seed):
    """Every call in any order, small pools that run out, repeated and bad ids: the device against the lists."""
    rng = np.random.default_rng([seed, page])
    n_pages, S, P = 30, 7, 9
    c = PagedCache(layers, n_pages, page, Hkv, dh, S, P, dtype=dtype)
    c.k.copy_(torch.randn(c.k.shape, device="cuda").to(dtype))
    c.v.copy_(torch.randn(c.v.shape, device="cuda").to(dtype))
    r = host_copy(c)
    c.reset()
    for step in range(60):
        n = int(rng.integers(1, S + 1))
        seqs = rng.permutation(S)[:n].tolist()
        if rng.random() < 0.15:
            seqs[-1] = int(rng.choice([-1, S, seqs[0]]))
        do = rng.choice(["grow", "grow", "grow", "path", "fork", "truncate", "compact"])
        if do in ("grow", "path"):
            rows = [int(x) for x in rng.integers(0, 2 * page + 3, n)]
            off = np.concatenate([[0], np.cumsum(rows)]).tolist()
            kn, vn = (torch.randn((layers, max(off[-1], 1), Hkv, dh), device="cuda").to(dtype) for _ in range(2))
            new = {(l, kv): x[l].float().cpu().numpy() for l in range(layers) for kv, x in enumerate((kn, vn))}
            path = acc = None
            if do == "path":
                most = max(max(rows), 1)
                path = [(sorted(rng.permutation(m)[:rng.integers(0, m + 1)].tolist()) + [-1] * most)[:most] for m in rows]
                acc = [sum(x >= 0 for x in p) for p in path]
                if rng.random() < 0.1:
                    acc[0] += 1
            if rng.random() < 0.9:
                grow = acc if do == "path" else rows
                c.reserve(dev(seqs), dev(grow))
                r.reserve(seqs, grow)
                same(c, r)
            kw = dict(path=dev(path), n_acc=dev(acc)) if do == "path" else {}
            c.append(dev(seqs), kn, vn, dev(off), **kw)
            r.append(seqs, off, new, path, acc)
        elif do == "fork":
            k = int(rng.integers(1, 4))
            ids = rng.permutation(S).tolist()
            src, dst = [ids[int(rng.integers(2))] for _ in range(k)], ids[2:2 + k]
            if rng.random() < 0.2:
                dst[0] = int(rng.choice([src[-1], -1, S, dst[-1]]))
            c.fork(dev(src), dev(dst))
            r.fork(src, dst)
        elif do == "truncate":
            lens = [int(rng.integers(-1, r.lens[s] + 2)) if 0 <= s < S else 0 for s in seqs]
            c.truncate(dev(seqs), dev(lens))
            r.truncate(seqs, lens)
        else:
            used = c.compact()
            assert used.item() == r.compact()
        same(c, r)
        c.status.zero_()
        r.status = 0


def test_a_large_pool_in_one_call():
    """More pages, entries and free ids than a planning block has threads."""
    rng = np.random.default_rng(5)
    S, P, page, n_pages = 2500, 6, 2, 9001
    c = PagedCache(1, n_pages, page, 1, 8, S, P, dtype=BF)
    r = host_copy(c)
    seqs = rng.permutation(S).tolist()
    grow = rng.integers(0, 8, S).tolist()
    c.reserve(dev(seqs), dev(grow))
    want, free = [[] for _ in range(S)], 0                              # (the lists' reserve takes minutes here)
    for s, g in zip(seqs, grow):
        m = -(-g // page)
        want[s] = list(range(free, free + m)) + [-1] * (P - m)
        free += m
    assert c.table.tolist() == want and c.status.item() == 0 and c.refs.sum().item() == free
    rows = torch.randn((1, sum(grow), 1, 8), device="cuda").to(BF)
    c.append(dev(seqs), rows, rows, dev(np.concatenate([[0], np.cumsum(grow)])))
    assert c.status.item() == 0 and [c.lens.tolist()[s] for s in seqs] == grow
    drop = seqs[::2]
    c.truncate(dev(drop), dev([0] * len(drop)))
    before = {s: c.table[s].tolist() for s in seqs[1::2][:50]}
    data = {s: c.k[0, [p for p in t if p >= 0]].clone() for s, t in before.items()}
    used = c.compact().item()
    held = c.table[c.table >= 0]
    assert used == held.numel() == (c.refs > 0).sum().item() and held.max().item() == used - 1 and (c.refs[:used] == 1).all()
    for s, t in before.items():
        assert torch.equal(c.k[0, c.table[s][c.table[s] >= 0].long()], data[s])


def test_a_run_of_the_calls_together():
    """A prompt, samples of it, verified trees whose paths are appended: every pass's attention against the positions so far."""
    rng = np.random.default_rng(6)
    torch.manual_seed(6)
    layers, Hkv, heads, dh, page, S = 2, 2, 4, 64, 4, 5
    c = PagedCache(layers, 60, page, Hkv, dh, S, 12, dtype=BF)
    kn, vn = (torch.randn((layers, 10, Hkv, dh), device="cuda").to(BF) for _ in range(2))
    c.reserve(dev([0]), dev([10]))
    c.append(dev([0]), kn, vn, dev([0, 10]))
    c.fork(dev([0, 0]), dev([1, 3]))
    seqs = [3, 1, 0]
    history = {s: (kn.clone(), vn.clone()) for s in seqs}
    for _ in range(4):
        nodes = rng.integers(1, 9, len(seqs)).tolist()
        trees = [random_tree(rng, n) for n in nodes]
        off = np.concatenate([[0], np.cumsum(nodes)])
        rows = int(off[-1])
        tokens, predicted = rng.integers(2, size=rows), rng.integers(2, size=rows)
        q = torch.randn((layers, rows, heads, dh), device="cuda").to(BF)
        kn, vn = (torch.randn((layers, rows, Hkv, dh), device="cuda").to(BF) for _ in range(2))
        parent = dev(sum(trees, []))
        for l in range(layers):
            out, lse = c.attention(l, q[l], kn[l], vn[l], dev(off), parent, seqs=dev(seqs), want_lse=True)
            for e, s in enumerate(seqs):
                a, b = int(off[e]), int(off[e + 1])
                k, v = (torch.cat([h[l], x[l, a:b]]).transpose(0, 1).double().cpu().numpy() for h, x in zip(history[s], (kn, vn)))
                n = history[s][0].shape[1]
                want, wl, to, tl = R.attention(q[l, a:b].double().cpu().numpy(), k, v, R.visible(trees[e], n, 0, 0), dh ** -0.5, UNIT[BF])
                assert (np.abs(out[a:b].double().cpu().numpy() - want) <= to).all()
        path, n_acc, _ = tree_accept(dev(tokens), parent, dev(off), dev(predicted))
        c.reserve(dev(seqs), n_acc)
        c.append(dev(seqs), kn, vn, dev(off), path=path, n_acc=n_acc)
        for e, s in enumerate(seqs):
            took, _ = R.accept(tokens[off[e]:off[e + 1]].tolist(), trees[e], predicted[off[e]:off[e + 1]].tolist())
            history[s] = tuple(torch.cat([h, x[:, int(off[e]):int(off[e + 1])][:, took]], 1) for h, x in zip(history[s], (kn, vn)))
        if rng.random() < 0.5:
            c.compact()
    c.check()


# ------------------------------------------------------------------------------------------ scores
def check_scores(x, tokens, top, got):
    lp, ent, rank, ids, tops = (t.cpu() for t in got)
    x = x.double().cpu()
    z = torch.log_softmax(x, 1)
    n, V = x.shape
    # the sum: its exponentials are off by 2^-22, its arguments by the rounding of a difference; terms are added in float32
    spread = (x.masked_fill(torch.isinf(x), 0).abs().max(1).values + 16).clamp(max=1e4)
    tol = 2.0 ** -21 + 2.0 ** -24 * spread + 2.0 ** -24 * min(V, 3000)
    t = tokens.long().cpu()
    ok = (t >= 0) & (t < V)
    at = torch.arange(n)[ok]
    want = z[at, t[ok]]
    same_inf = torch.isinf(want)
    assert torch.equal(torch.isinf(lp[ok]), same_inf)
    assert ((lp[ok].double() - want).abs() <= tol[ok] + 2.0 ** -22 * want.abs())[~same_inf].all()
    assert (rank[ok] == (x[at] > x[at, t[ok]][:, None]).sum(1).int()).all()
    assert torch.isneginf(lp[~ok]).all() and (rank[~ok] == -1).all()
    h = -(z.exp() * z.masked_fill(torch.isinf(z), 0)).sum(1)
    assert ((ent.double() - h).abs() <= tol * (1 + h)).all(), float(((ent.double() - h).abs() / tol).max())
    order = (x + 0.0).sort(dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(ids.long(), order)
    want = z.gather(1, order)
    fin = ~torch.isinf(want)
    assert torch.equal(torch.isinf(tops), ~fin)
    assert ((tops.double() - want).abs() <= tol[:, None] + 2.0 ** -22 * want.abs())[fin].all()


@pytest.mark.parametrize("dtype", [torch.float32, BF, HF])
@pytest.mark.parametrize("vocab", [1, 2, 7, 31, 33, 131, 1027, 2048, 2049, 5003, 50001])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_scores(dtype, vocab, top):
    torch.manual_seed(vocab + top)
    rows = 9
    x = (torch.randn((rows, vocab), device="cuda") * torch.tensor([0.01, 1, 2, 3, 5, 8, 1, 1, 20], device="cuda")[:, None]).to(dtype)
    x[6].masked_fill_(torch.rand(vocab, device="cuda") < 0.5, float("-inf"))
    x[6, 0] = 0.0
    x[7] = x[7].sort().values                                            # rising: every value enters
    t = torch.randint(vocab, (rows,), device="cuda", dtype=torch.int32)
    t[6], t[3], t[4] = 0, -1, vocab
    check_scores(x, t, min(top, vocab), logprobs(x, t, top=min(top, vocab)))


@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 3), (3, 5), (7, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, BF])
def test_scores_of_rows_that_lie_apart(offset, pad, dtype):
    torch.manual_seed(offset)
    big = torch.randn((6, 1027 + offset + pad), device="cuda").to(dtype)
    x = big[:, offset:offset + 1027]
    t = torch.randint(1027, (6,), device="cuda", dtype=torch.int32)
    check_scores(x, t, 8, logprobs(x, t, top=8))


def test_scores_of_equal_values_and_signed_zeros():
    x = torch.zeros((2, 100), device="cuda")
    x[0, ::2] = -0.0
    x[1, 40:] = 1.0
    got = logprobs(x, dev([5, 3]), top=20)
    check_scores(x, dev([5, 3]), 20, got)
    assert got[3][0].tolist() == list(range(20)) and got[3][1].tolist() == list(range(40, 60))


def test_scores_at_the_edges_of_the_types():
    inf, nan = float("inf"), float("nan")
    lowest = torch.finfo(torch.float32).min
    x = torch.randn((7, 300), device="cuda")
    x[0] = -inf
    x[1, 3] = inf
    x[2, 4] = nan
    x[3] = lowest
    x[4, 1:] = lowest
    x[5] = nan
    x[6, 2:] = -inf
    lp, ent, rank, ids, tops = (t.cpu() for t in logprobs(x, dev([0, 0, 0, 0, 0, 0, 0]), top=4))
    assert lp[0] == -inf and ent[0] == 0 and rank[0] == 0 and ids[0].tolist() == [0, 1, 2, 3] and torch.isneginf(tops[0]).all()
    assert torch.isnan(lp[1]) and torch.isnan(ent[1]) and ids[1, 0] == 3 and rank[1] == (x[1] > x[1, 0]).sum().cpu()
    assert torch.isnan(lp[2]) and torch.isnan(ent[2]) and torch.isnan(tops[2]).all() and 4 not in ids[2].tolist()
    assert abs(lp[3] + np.log(300)) < 1e-5 and abs(ent[3] - np.log(300)) < 1e-5
    assert abs(lp[4]) < 1e-6 and abs(ent[4]) < 1e-6 and ids[4].tolist() == [0, 1, 2, 3] and tops[4, 1] < -1e38
    assert torch.isnan(lp[5]) and rank[5] == 0 and ids[5].tolist() == [0, 1, 2, 3]
    assert torch.isneginf(tops[6, 2:]).all() and set(ids[6].tolist()) == {0, 1, 2, 3}


def test_scores_without_tokens_and_without_rows():
    x = torch.randn((3, 50), device="cuda")
    lp, ent, rank, ids, tops = logprobs(x)
    assert torch.isneginf(lp).all() and (rank == -1).all() and ids.shape == (3, 0)
    assert [t.shape[0] for t in logprobs(x[:0], top=3)] == [0] * 5


@pytest.mark.parametrize("rows,vocab", [(1, 150000), (3, 128011), (700, 1027), (40000, 40)])
def test_scores_of_few_and_of_many_rows(rows, vocab):
    torch.manual_seed(rows)
    x = torch.randn((rows, vocab), device="cuda").to(BF)
    t = torch.randint(vocab, (rows,), device="cuda", dtype=torch.int32)
    check_scores(x, t, 6, logprobs(x, t, top=6))


@pytest.mark.parametrize("page", [2, 4, 6, 8, 12, 20, 24, 36, 40, 48, 72, 96, 100, 160, 200])
@pytest.mark.parametrize("dh", [64, 128])
def test_pages_that_chunks_do_not_divide(page, dh):
    run_case(41, [0, 7, 8, 200, 777], [3, 1, 5, 2, 7], 4, 2, dh, page, BF)
    run_case(42, [500, 130], [20, 3], 2, 1, dh, page, HF, window=100, prefix=30)


@pytest.mark.parametrize("dh,nodes", [(64, 40), (128, 20), (64, 256), (128, 130)])
def test_trees_of_several_small_tiles(dh, nodes):
    run_case(43, [1500, 3, 260], [nodes, 1, nodes - 3], 3, 1, dh, 64, BF)
    run_case(44, [1500], [nodes], 2, 2, dh, 16, HF, window=400, prefix=70)


@pytest.mark.parametrize("dtype", [torch.float32, BF, HF])
@pytest.mark.parametrize("offset", [-60000.0, -8193.0, -8192.0, -700.0, 5.3, 8190.0, 8300.0, 50000.0])
def test_scores_far_from_zero(dtype, offset):
    """The form of the differences changes with the maximum; also where it rises past the change inside a row, and from -inf."""
    torch.manual_seed(int(offset))
    x = torch.randn((6, 9001), device="cuda") * 3 + offset
    x[1] = torch.linspace(offset - 900, offset + 900, 9001, device="cuda")
    x[2] = torch.linspace(offset + 900, offset - 900, 9001, device="cuda")
    x[3, :8000] = float("-inf")
    x[4, ::3] = -65504.0 if dtype is HF else -1e30
    x[5, 4500:] += 60 if dtype is HF else 3e4
    x = x.to(dtype)
    tokens = dev([0, 9000, 17, 8500, 3, 4600])
    for top in (0, 20):
        check_scores(x, tokens, top, logprobs(x, tokens, top=top))


@pytest.mark.parametrize("captured", [False, True])
def test_calls_that_follow_one_another_see_what_the_last_one_wrote(captured):
    """Launches are resident before the one in front ends; lengths, tables, references and rows still arrive.  Twelve positions, one or two a
    round, through acceptance, reservation, append, attention, fork and truncation, against the same rounds one at a time."""
    def rounds(c, wait):
        torch.manual_seed(5)
        i32 = dict(dtype=torch.int32, device="cuda")
        seqs, other, off = torch.arange(6, **i32), torch.arange(6, 12, **i32), dev(np.arange(7) * 4)
        parent, tokens, pred = dev([-1, 0, 1, 2] * 6), dev([1, 2, 3, 4] * 6), dev([2, 3, 4, 5] * 6)
        stop = torch.zeros(6, **i32)
        rows = [[torch.randn((n, 24, 2, 64), device="cuda").to(BF) for n in (3, 3, 1)] for _ in range(12)]
        q = [torch.randn((24, 4, 64), device="cuda").to(BF) for _ in range(12)]

        def go():
            out = []
            for (k, v, _), x in zip(rows, q):
                path, n, nxt = tree_accept(tokens, parent, off, pred, max_nodes=4); wait()
                c.reserve(seqs, n); wait()
                c.append(seqs, k, v, off, path, n); wait()
                for layer in range(3):
                    out += c.attention(layer, x, k[layer], v[layer], off, parent, seqs=seqs, max_nodes=4, want_lse=True); wait()
                c.fork(seqs, other); wait()
                out += c.attention(1, x, k[1], v[1], off, parent, seqs=other, max_nodes=4, want_lse=True); wait()
                out += logprobs(out[-2].flatten(1), tokens, top=3); wait()
                out += [nxt, c.lens.clone(), c.table.clone(), c.refs.clone(), c.compact()]; wait()
                c.truncate(other, stop); wait()
            return out
        return go

    def pool():
        c = PagedCache(3, 90, 4, 2, 64, 12, 14)
        c.reset()
        return c
    a, b = pool(), pool()
    want = rounds(a, torch.cuda.synchronize)()
    go = rounds(b, lambda: None)
    if captured:
        side = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                got = go()
            for _ in range(3):
                b.reset()
                g.replay()
    else:
        go()
        b.reset()
        got = go()
    torch.cuda.synchronize()
    a.check(), b.check()
    assert all(torch.equal(x, y) for x, y in zip(want, got)) and torch.equal(a.lens, b.lens) and int(b.lens[0]) == 48


def plain_tree(c, b, n, tree, q, kn, vn, window=0, prefix=0):
    k, v = gathered(c, 0, b, n, kn, vn)
    return R.attention(q.double().cpu().numpy(), k, v, R.visible(tree, n, window, prefix), c.head_dim ** -0.5, UNIT[c.dtype])


@pytest.mark.parametrize("dh", [64, 128])
def test_one_sequence_in_several_trees_and_bounded_positions(dh):
    rng = np.random.default_rng(51)
    c = filled(rng, [300, 90], 2, dh, 16, BF)
    trees = [random_tree(rng, n) for n in (5, 9, 1, 30)]
    seqs, rows = [0, 0, 1, 0], 45
    q, kn, vn = (torch.randn((rows, h, dh), device="cuda").to(BF) for h in (4, 2, 2))
    off = np.concatenate([[0], np.cumsum([len(t) for t in trees])])
    for most in (1600, 300, 137, 1, 0):
        out, lse = c.attention(0, q, kn, vn, dev(off), dev(sum(trees, [])), seqs=dev(seqs), max_len=most, want_lse=True)
        for i, (b, tree) in enumerate(zip(seqs, trees)):
            at = slice(off[i], off[i + 1])
            want, wl, to, tl = plain_tree(c, b, min([300, 90][b], most), tree, q[at], kn[at], vn[at])
            assert (np.abs(out[at].double().cpu().numpy() - want) <= to).all()
            live = ~np.isneginf(wl)
            got = lse[at].double().cpu().numpy()
            assert (np.isneginf(got) == ~live).all() and (np.abs(got[live] - wl[live]) <= tl[live]).all()
    c.check()


def test_the_most_trees_and_one_more():
    n = 513
    c = PagedCache(1, n, 16, 1, 64, n, 1)
    c.reset()
    seqs = torch.arange(n, dtype=torch.int32, device="cuda")
    c.reserve(seqs, seqs % 17)
    c.lens.copy_(seqs % 17)
    c.k.normal_(), c.v.normal_()
    c.check()
    q, kn, vn = (torch.randn((n, 1, 64), device="cuda").to(BF) for _ in range(3))
    parent = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    out = c.attention(0, q[:512], kn[:512], vn[:512], torch.arange(513, dtype=torch.int32, device="cuda"), parent[:512], max_nodes=1)
    for b in (0, 1, 15, 16, 17, 300, 511):
        want, _, to, _ = plain_tree(c, b, b % 17, [-1], q[b:b + 1], kn[b:b + 1], vn[b:b + 1])
        assert (np.abs(out[b:b + 1].double().cpu().numpy() - want) <= to).all()
    with pytest.raises(FmError) as e:
        c.attention(0, q, kn, vn, torch.arange(n + 1, dtype=torch.int32, device="cuda"), parent, max_nodes=1)
    assert e.value.code == -3


def test_calls_on_a_stream_follow_what_is_enqueued_there():
    rng = np.random.default_rng(52)
    c = filled(rng, [200], 2, 64, 16, BF)
    q, kn, vn = (torch.randn((3, h, 64), device="cuda").to(BF) for h in (4, 2, 2))
    off, parent = dev([0, 3]), dev([-1, 0, 0])
    want = c.attention(0, q, kn, vn, off, parent)
    x, t = torch.randn((3, 5000), device="cuda"), dev([1, 2, 3])
    scores = logprobs(x, t, top=4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late, late_x = torch.zeros_like(q), torch.zeros_like(x)
        torch.cuda._sleep(20_000_000)                                     # (10 ms)
        late.copy_(q), late_x.copy_(x)
        got, got_scores = c.attention(0, late, kn, vn, off, parent), logprobs(late_x, t, top=4)
    side.synchronize()
    assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(got_scores, scores))
