"""Performance cases of the operators for trees of drafts over a paged cache, through their public Python entry points.

A case names an operator (`do`) and its sizes:

  attend    attention of a tree of drafted tokens over the pages of each sequence's cache (one node: a single token)
  commit    what follows a verified tree: the longest accepted path, pages for it, its keys and values into every layer's cache
  branch    several continuations of one sequence: fork, pages of their own (a shared last page is copied), a first append
  turnover  finished sequences give their pages back and the pool is compacted for what remains
  score     log probabilities of given tokens with entropy, rank and top alternatives

`own` false computes the plain form in elementary torch operations; true calls the framework.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _attend(name, batch, heads, kv_heads, dim, page, length, length_to, nodes, nodes_to, window=0, prefix=0, dtype="bf16"):
    return {"name": name, "do": "attend", "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "length": length,
            "length_to": length_to, "nodes": nodes, "nodes_to": nodes_to, "window": window, "prefix": prefix, "dtype": dtype}


def _pages(name, do, batch, layers, kv_heads, dim, page, length, length_to, nodes, dtype="bf16"):
    return {"name": name, "do": do, "batch": batch, "layers": layers, "kv_heads": kv_heads, "dim": dim, "page": page, "length": length,
            "length_to": length_to, "nodes": nodes, "dtype": dtype}


def _score(name, rows, vocab, top, dtype, masked=False):
    return {"name": name, "do": "score", "rows": rows, "vocab": vocab, "top": top, "dtype": dtype, "masked": masked}


def listed():
    return [
        # the smallest verification: main token and three drafts of the tiny model behind its 64 conditioning slots
        _attend("tiny tree", 1, 4, 4, 64, 16, 150, 150, 4, 4),
        # the medium model's coordinate level deep in a mesh: 28 candidates, a window of 8192, 512 conditioning slots
        _attend("tree in a long mesh", 1, 16, 16, 64, 64, 20000, 20000, 28, 28, window=8192, prefix=512),
        # serving a batch one token at a time, grouped heads, small pages
        _attend("single tokens", 64, 32, 8, 128, 16, 100, 8000, 1, 1, dtype="fp16"),
        # wide trees over long ragged caches, grouped heads: as much arithmetic as memory traffic
        _attend("wide trees, long caches", 8, 32, 8, 128, 64, 20000, 32768, 33, 64),
        # one sequence of the medium model accepts a path of a small tree: latency
        _pages("commit of one", "commit", 1, 32, 16, 64, 64, 700, 700, 10),
        # the same for the batched model
        _pages("commit of a batch", "commit", 16, 32, 16, 64, 64, 585, 9000, 28),
        # four samples from one prompt of the small model
        _pages("four samples", "branch", 1, 14, 8, 64, 16, 329, 329, 4),
        # several samples of every sequence of a batch
        _pages("samples of a batch", "branch", 16, 32, 16, 64, 64, 585, 2000, 6),
        # a small pool after a few requests have ended
        _pages("small turnover", "turnover", 8, 14, 8, 64, 16, 73, 700, 0),
        # a serving pool half of whose sequences have ended
        _pages("pool turnover", "turnover", 32, 32, 16, 64, 64, 100, 2400, 0),
        # scores of one pass's ten rows over the mesh vocabulary: latency
        _score("rows of a pass", 10, 1027, 4, "fp32"),
        # scoring a batch of text positions over a large vocabulary with some tokens forbidden
        _score("large vocabulary", 512, 128011, 20, "bf16", masked=True),
    ]


def draw(rng):
    """One more case of these ranges, without a name."""
    case = _drawn(rng)
    del case["name"]
    return case


def _drawn(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    do = rng.choice(["attend", "attend", "attend", "commit", "branch", "turnover", "score", "score"])
    if do == "score":
        vocab = log_int(100, 150000)
        return _score(None, log_int(1, max(1, min(40000, 60000000 // vocab))), vocab, rng.choice([0, 1, 4, 5, 20, 32]), rng.choice(["bf16", "fp16", "fp32"]),
                      rng.random() < 0.4)
    dim, page, dtype = rng.choice([64, 64, 128]), rng.choice([8, 16, 24, 32, 64, 64, 128, 100]), rng.choice(["bf16", "bf16", "fp16"])
    if do == "attend":
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        group = rng.choice([1, 1, 2, 4, 7, 8])
        batch = log_int(1, 64)
        most = max(16, min(40000, 180000 * 1024 // (batch * kv_heads * dim)))
        length_to = log_int(1, most)
        nodes_to = log_int(1, max(1, min(256, 64 * 8 * 32 * 32768 // (batch * kv_heads * group * length_to))))
        return _attend(None, batch, kv_heads * group, kv_heads, dim, page, log_int(1, length_to), length_to, log_int(1, nodes_to), nodes_to,
                       window=rng.choice([0, 0, 0, log_int(1, 8192)]), prefix=rng.choice([0, 0, 64, 512]), dtype=dtype)
    kv_heads, layers, batch = rng.choice([1, 2, 4, 8, 16]), rng.randint(1, 32), log_int(1, 32)
    most = max(16, min(9000, 2500000000 // (batch * kv_heads * dim * layers * 4)))
    length_to = log_int(10, most)
    return _pages(None, do, batch, layers, kv_heads, dim, page, log_int(1, length_to), length_to, rng.randint(1, 40) if do == "commit" else rng.randint(1, 6),
                  dtype=dtype)


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _ragged(case, n, lo, hi):
    """n sizes spread over [lo, hi], the largest among them: the case's own, whatever the seed."""
    rng = np.random.default_rng([n, lo, hi, case["page"]])
    x = np.exp(rng.uniform(math.log(max(lo, 1)), math.log(hi + 1), n)).astype(np.int64)
    x = np.clip(x, lo, hi)
    x[rng.integers(n)] = hi
    return x


def _parents(rng, counts):
    """Trees as drafting makes them: long runs with branches; now and then a node that was pruned (-2)."""
    out = []
    for n in counts:
        i = np.arange(n)
        p = np.where(rng.random(n) < 0.6, i - 1, (rng.random(n) * np.maximum(i, 1)).astype(np.int64))
        p = np.where(rng.random(n) < 0.03, -2, p)
        p[0] = -1
        out.append(p)
    return np.concatenate(out)


def _dev(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x)).to(device="cuda", dtype=dtype)


def _pool(rng, case, layers, lens, spare, max_pages, max_seqs):
    """A pool in use: the sequences' pages lie in any order, some pages are free."""
    page = case["page"]
    have = -(-np.asarray(lens) // page)
    n_pages = int(have.sum()) + spare
    order = rng.permutation(n_pages)
    table, refs, at = np.full((max_seqs, max_pages), -1, np.int64), np.zeros(n_pages, np.int64), 0
    for b, n in enumerate(have):
        table[b, :n] = order[at:at + n]
        at += n
    refs[order[:at]] = 1
    shape = (layers, n_pages, case["kv_heads"], page, case["dim"])
    k, v = (torch.randn(shape, device="cuda", dtype=_TYPES[case["dtype"]]) for _ in range(2))
    full = np.zeros(max_seqs, np.int64)
    full[:len(lens)] = lens
    return SimpleNamespace(k=k, v=v, table=_dev(table), lens=_dev(full), refs=_dev(refs))


def _handle(s):
    """The object through which a program of the framework's user holds the pool."""
    from paper_2511_15618_b200 import PagedCache
    return PagedCache.over(s.k, s.v, table=s.table, lens=s.lens, refs=s.refs)


def prepare(case, seed):
    rng = np.random.default_rng([seed, 5])
    torch.manual_seed(seed)
    do = case["do"]
    if do == "score":
        dtype = _TYPES[case["dtype"]]
        x = torch.randn((case["rows"], case["vocab"]), device="cuda") * 2.0
        tokens = _dev(rng.integers(case["vocab"], size=case["rows"]))
        # a trained model is often sure: the given token or another stands out in most rows
        x[torch.arange(case["rows"], device="cuda"), _dev(rng.integers(case["vocab"], size=case["rows"]), torch.int64)] += _dev(rng.uniform(0, 18, case["rows"]), torch.float32)
        if case["masked"]:
            x.masked_fill_(torch.rand((1, case["vocab"]), device="cuda") < 0.25, float("-inf"))
            x[:, 0] = 0.5
            tokens = torch.where(torch.isinf(x[torch.arange(case["rows"], device="cuda"), tokens.long()]), torch.zeros_like(tokens), tokens)
        return SimpleNamespace(do=do, logits=x.to(dtype), tokens=tokens, top=case["top"])
    B, page, dtype = case["batch"], case["page"], _TYPES[case["dtype"]]
    lens = _ragged(case, B, case["length"], case["length_to"])
    if do == "attend":
        counts = _ragged(case, B, case["nodes"], case["nodes_to"])
        rows = int(counts.sum())
        max_pages = -(-int(lens.max()) // page)
        s = _pool(rng, case, 1, lens, 3, max_pages, B)
        s.q = torch.randn((rows, case["heads"], case["dim"]), device="cuda").mul_(1.5).to(dtype)
        s.k_new, s.v_new = (torch.randn((rows, case["kv_heads"], case["dim"]), device="cuda").to(dtype) for _ in range(2))
        s.row_off = _dev(np.concatenate([[0], np.cumsum(counts)]))
        s.parent = _dev(_parents(rng, counts))
        s.window, s.prefix, s.max_nodes, s.max_len = case["window"], case["prefix"], int(counts.max()), int(lens.max())
    elif do == "commit":
        counts = np.full(B, case["nodes"])
        rows = int(counts.sum())
        max_pages = -(-(int(lens.max()) + case["nodes"]) // page)
        s = _pool(rng, case, case["layers"], lens, B * (case["nodes"] // page + 2), max_pages, B)
        s.seqs, s.base = _dev(np.arange(B)), s.lens.clone()
        s.k_new, s.v_new = (torch.randn((case["layers"], rows, case["kv_heads"], case["dim"]), device="cuda").to(dtype) for _ in range(2))
        s.row_off = _dev(np.concatenate([[0], np.cumsum(counts)]))
        parent = _parents(rng, counts)
        s.parent = _dev(parent)
        # predictions that agree with a draft most of the time, as those of a trained draft module do
        tokens = rng.integers(8, size=rows)
        first = np.repeat(np.cumsum(counts) - counts, counts)
        predicted = rng.integers(8, size=rows)
        hit = (parent >= 0) & (rng.random(rows) < 0.75)
        predicted[(first + parent)[hit]] = tokens[hit]
        s.tokens, s.predicted, s.max_nodes = _dev(tokens), _dev(predicted), case["nodes"]
        s.grow = _dev(counts)
    elif do == "branch":
        copies, new = case["nodes"], 1
        n_dst = B * copies
        max_pages = int(lens.max()) // page + 2
        s = _pool(rng, case, case["layers"], lens, 2 * (n_dst + B) + 2, max_pages, B + n_dst)
        s.src, s.dst = _dev(np.repeat(np.arange(B), copies)), _dev(B + np.arange(n_dst))
        s.sources, s.base = _dev(np.arange(B)), s.lens[:B].clone()
        # the copies come first: the last holder of a shared page, the source, then keeps it
        s.seqs = _dev(np.concatenate([B + np.arange(n_dst), np.arange(B)]))
        rows = n_dst + B
        s.k_new, s.v_new = (torch.randn((case["layers"], rows, case["kv_heads"], case["dim"]), device="cuda").to(dtype) for _ in range(2))
        s.row_off = _dev(np.arange(rows + 1))
        s.grow = _dev(np.full(rows, new))
    else:
        max_pages = -(-int(lens.max()) // page)
        s = _pool(rng, case, case["layers"], lens, max(2, int(lens.sum()) // page // 8), max_pages, B)
        s.seqs = _dev(rng.permutation(B)[:(B + 1) // 2])
        s.nothing = torch.zeros_like(s.seqs)
        s.table0, s.refs0, s.lens0 = s.table.clone(), s.refs.clone(), s.lens.clone()
    s.do, s.page = do, page
    s.cache = _handle(s) if own else None
    return s


# ------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------
def _plain_trees(row_off, parent, n_max):
    """Padded rows [B, n_max], which of them are nodes, and reach[b, i, j]: j is i or an ancestor of i (live nodes only)."""
    first = row_off[:-1].long()[:, None]
    i = torch.arange(n_max, device=parent.device)
    there = i < (row_off[1:].long()[:, None] - first)
    rows = torch.where(there, first + i, first.clamp(max=parent.numel() - 1))
    p = torch.where(there, parent[rows].long(), -2)
    good = (p >= 0) & (p < i)
    edge = torch.zeros(p.shape + (n_max,), device=parent.device)
    edge.scatter_(2, p.clamp(0, n_max - 1)[..., None], good[..., None].float())
    eye = torch.eye(n_max, device=parent.device).expand_as(edge)
    # (I - A)^-1 = I + A + A^2 + ...: one entry for each ancestor
    reach = torch.linalg.solve_triangular(eye - edge, eye.contiguous(), upper=False) > 0.5
    dead = ~(good | (p == -1))
    live = there & ~(reach & dead[:, None, :]).any(2)
    return rows, there, p, reach & live[:, :, None] & live[:, None, :], live


def _plain_attend(s):
    B, page = s.row_off.numel() - 1, s.page
    n_max, (rows_all, H, dh), Hkv = s.max_nodes, s.q.shape, s.k.shape[2]
    G = H // Hkv
    rows, there, p, reach, live = _plain_trees(s.row_off, s.parent, n_max)
    q = s.q[rows].float().view(B, n_max, Hkv, G, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n_max, dh)
    take = s.table.long().clamp(min=0)
    S = take.shape[1] * page

    def context(pool):
        return pool[0][take].permute(0, 2, 1, 3, 4).reshape(B, Hkv, S, dh).float()

    def drafted(x):
        return x[rows].float().permute(0, 2, 1, 3)

    scale = 1.0 / math.sqrt(dh)
    old = torch.matmul(q, context(s.k).transpose(2, 3)).mul_(scale).view(B, Hkv, G, n_max, S)
    new = torch.matmul(q, drafted(s.k_new).transpose(2, 3)).mul_(scale).view(B, Hkv, G, n_max, n_max)
    slot = torch.arange(S, device=q.device)
    length = s.lens.long()[:, None, None]
    depth = reach.sum(2) - 1
    see = (slot < length) & live[:, :, None]
    if s.window > 0:
        see = see & ((slot < s.prefix) | (length + depth[:, :, None] - slot < s.window))
        reach = reach & (depth[:, :, None] - depth[:, None, :] < s.window)
    old.masked_fill_(~see[:, None, None], float("-inf"))
    new.masked_fill_(~reach[:, None, None], float("-inf"))
    top = torch.maximum(old.amax(-1), new.amax(-1))
    base = torch.where(torch.isinf(top), torch.zeros_like(top), top)[..., None]
    old, new = old.sub_(base).exp_(), new.sub_(base).exp_()
    total = old.sum(-1) + new.sum(-1)
    lse = torch.where(total > 0, base[..., 0] + total.log(), float("-inf"))
    out = torch.matmul(old.view(B, Hkv, G * n_max, S), context(s.v)) + torch.matmul(new.view(B, Hkv, G * n_max, n_max), drafted(s.v_new))
    out = (out.view(B, Hkv, G, n_max, dh) / total.clamp(min=1e-30)[..., None]).permute(0, 3, 1, 2, 4).reshape(B, n_max, H, dh)
    lse = lse.permute(0, 3, 1, 2).reshape(B, n_max, H)
    return out[there].to(s.q.dtype), lse[there]


def _plain_accept(s):
    rows, there, p, reach, live = _plain_trees(s.row_off, s.parent, s.max_nodes)
    i = torch.arange(s.max_nodes, device=p.device)
    token, predicted = s.tokens[rows], s.predicted[rows]
    match = live & (p >= 0) & (token == predicted.gather(1, p.clamp(min=0)))
    sibling = (p[:, :, None] == p[:, None, :]) & match[:, None, :] & (i[None, :] < i[:, None])
    chosen = (match & ~sibling.any(2)) | (i == 0)
    taken = live & ~(reach & ~chosen[:, None, :]).any(2) & (reach[:, :, 0] | (i == 0))
    n_acc = taken.sum(1)
    order = torch.where(taken, i, s.max_nodes).sort(1).values
    path = torch.where(order < s.max_nodes, order, -1)
    last = path.gather(1, (n_acc - 1).clamp(min=0)[:, None])
    next_token = torch.where(n_acc > 0, predicted.gather(1, last.clamp(min=0))[:, 0], -1)
    return path.int(), n_acc.int(), next_token.int()


def _plain_truncate(s, seqs, lens):
    seqs = seqs.long()
    left = torch.minimum(s.lens[seqs], lens.clamp(min=0))
    t = s.table[seqs]
    drop = (torch.arange(t.shape[1], device=t.device) >= (left[:, None] + s.page - 1) // s.page) & (t >= 0)
    s.refs.index_add_(0, t[drop].long(), torch.full_like(t[drop], -1))
    s.table[seqs] = torch.where(drop, -1, t)
    s.lens[seqs] = left


def _plain_reserve(s, seqs, grow):
    seqs = seqs.long()
    length, t = s.lens[seqs].long(), s.table[seqs].long()
    j = torch.arange(t.shape[1], device=t.device)
    last = length // s.page
    held = t.gather(1, last.clamp(max=t.shape[1] - 1)[:, None])[:, 0]
    same = torch.tril((held[:, None] == held[None, :]) & (length % s.page > 0)[None, :], -1)
    split = (length % s.page > 0) & (grow > 0) & (held >= 0) & (s.refs[held.clamp(min=0)] - same.sum(1) > 1)
    want = (j < ((length + grow + s.page - 1) // s.page)[:, None]) & ((t < 0) | ((j == last[:, None]) & split[:, None]))
    ids = (s.refs == 0).nonzero()[:int(want.sum()), 0]
    fresh = t.clone()
    fresh[want] = ids
    old, new = held[split], fresh.gather(1, last.clamp(max=t.shape[1] - 1)[:, None])[:, 0][split]
    keep = (torch.arange(s.page, device=t.device) < (length % s.page)[split][:, None])[None, :, None, :, None]
    s.k[:, new] = torch.where(keep, s.k[:, old], s.k[:, new])
    s.v[:, new] = torch.where(keep, s.v[:, old], s.v[:, new])
    s.refs.index_add_(0, old, torch.full_like(old, -1, dtype=torch.int32))
    s.refs[ids] = 1
    s.table[seqs] = fresh.int()


def _plain_append(s, seqs, path=None, n_acc=None):
    seqs = seqs.long()
    n = n_acc.long() if n_acc is not None else (s.row_off[1:] - s.row_off[:-1]).long()
    most = path.shape[1] if path is not None else 1
    j = torch.arange(most, device=n.device)
    take = j < n[:, None]
    rows = (s.row_off[:-1].long()[:, None] + (path.long() if path is not None else j))[take]
    slot = s.lens[seqs].long()[:, None] + j
    page = s.table[seqs].long().gather(1, (slot // s.page).clamp(max=s.table.shape[1] - 1))[take]
    at = (slot % s.page)[take]
    s.k[:, page, :, at] = s.k_new[:, rows].transpose(0, 1)
    s.v[:, page, :, at] = s.v_new[:, rows].transpose(0, 1)
    s.lens[seqs] += n.int()


def _plain_fork(s, src, dst):
    src, dst = src.long(), dst.long()
    t = s.table[dst]
    s.refs.index_add_(0, t[t >= 0].long(), torch.full_like(t[t >= 0], -1))
    t = s.table[src]
    s.refs.index_add_(0, t[t >= 0].long(), torch.ones_like(t[t >= 0]))
    s.table[dst] = t
    s.lens[dst] = s.lens[src]


def _plain_compact(s):
    used = s.refs > 0
    n = used.sum()
    i = torch.arange(used.numel(), device=used.device)
    old, new = ((i >= n) & used).nonzero()[:, 0], ((i < n) & ~used).nonzero()[:, 0]
    s.k[:, new] = s.k[:, old]
    s.v[:, new] = s.v[:, old]
    goes = i.int()
    goes[old] = new.int()
    s.table.copy_(torch.where(s.table >= 0, goes[s.table.clamp(min=0).long()], s.table))
    s.refs[new] = s.refs[old]
    s.refs[old] = 0
    return n.int().view(1)


def _plain_score(s):
    x = s.logits.float() + 0.0
    t = s.tokens.long()[:, None]
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(1, keepdim=True)
    given = x.gather(1, t)
    logprob = (given - top) - total.log()
    entropy = total.log() - torch.where(e > 0, (x - top) * e, 0.0).sum(1, keepdim=True) / total
    rank = (x > given).sum(1)
    bits = x.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + ((1 << 32) - 1 - torch.arange(x.shape[1], device=x.device))
    ids = key.topk(s.top, 1).indices
    return logprob[:, 0], entropy[:, 0], rank.int(), ids.int(), (x.gather(1, ids) - top) - total.log()


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(s):
    if s.do == "score":
        if own:
            from paper_2511_15618_b200 import logprobs
            return logprobs(s.logits, s.tokens, top=s.top)
        return _plain_score(s)
    if s.do == "attend":
        if own:
            return s.cache.attention(0, s.q, s.k_new, s.v_new, s.row_off, s.parent, window=s.window, n_prefix=s.prefix, max_nodes=s.max_nodes,
                                     max_len=s.max_len, want_lse=True)
        return _plain_attend(s)
    if s.do == "commit":
        # the sequences go back to where the last pass began, as after a rejected continuation
        if own:
            from paper_2511_15618_b200 import tree_accept
            s.cache.truncate(s.seqs, s.base)
            path, n_acc, next_token = tree_accept(s.tokens, s.parent, s.row_off, s.predicted, max_nodes=s.max_nodes)
            s.cache.reserve(s.seqs, n_acc)
            s.cache.append(s.seqs, s.k_new, s.v_new, s.row_off, path=path, n_acc=n_acc)
        else:
            _plain_truncate(s, s.seqs, s.base)
            path, n_acc, next_token = _plain_accept(s)
            _plain_reserve(s, s.seqs, n_acc)
            _plain_append(s, s.seqs, path, n_acc)
        return path, n_acc, next_token, s.k, s.v, s.table, s.lens, s.refs
    if s.do == "branch":
        if own:
            s.cache.truncate(s.sources, s.base)
            s.cache.fork(s.src, s.dst)
            s.cache.reserve(s.seqs, s.grow)
            s.cache.append(s.seqs, s.k_new, s.v_new, s.row_off, max_rows=1)
        else:
            _plain_truncate(s, s.sources, s.base)
            _plain_fork(s, s.src, s.dst)
            _plain_reserve(s, s.seqs, s.grow)
            _plain_append(s, s.seqs)
        return s.k, s.v, s.table, s.lens, s.refs
    # a pool in use again, as the next requests leave it
    s.table.copy_(s.table0)
    s.refs.copy_(s.refs0)
    s.lens.copy_(s.lens0)
    if own:
        s.cache.truncate(s.seqs, s.nothing)
        used = s.cache.compact()
    else:
        _plain_truncate(s, s.seqs, s.nothing)
        used = _plain_compact(s)
    return used, s.k, s.v, s.table, s.lens, s.refs


# ------------------------------------------------------------------------------------------
# what a pass cannot do without, and its exact outputs
# ------------------------------------------------------------------------------------------
def work(case):
    """Expected sizes: ragged ones at the mean of their distribution."""
    def mean(lo, hi):
        return float(hi) if hi <= lo else (hi - lo) / math.log((hi + 1) / max(lo, 1))

    do = case["do"]
    if do == "score":
        n, size = case["rows"] * case["vocab"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": n * size + case["rows"] * (16 + 8 * case["top"]), "flops": 4.0 * n}
    B, length = case["batch"], mean(case["length"], case["length_to"])
    token = case["kv_heads"] * case["dim"] * 2 * 2                     # bytes of a position's keys and values in a layer
    if do == "attend":
        nodes = mean(case["nodes"], case["nodes_to"])
        seen = length if case["window"] == 0 else min(length, case["window"] + case["prefix"])
        rows = B * nodes
        return {"bytes": B * (seen + nodes) * token + rows * case["heads"] * (4 * case["dim"] + 4) + rows * 4,
                "flops": 4.0 * rows * case["heads"] * case["dim"] * (seen + nodes / 2)}
    table = 4.0 * B * length / case["page"]
    if do == "commit":
        return {"bytes": 2 * B * min(4.0, case["nodes"]) * token * case["layers"] + B * case["nodes"] * 12, "flops": 0}
    if do == "branch":
        n_dst = B * case["nodes"]
        return {"bytes": 2 * token * case["layers"] * (n_dst * case["page"] / 2 + n_dst + B) + table * (1 + 2 * case["nodes"]), "flops": 0}
    moved = B * length / 4 / case["page"] + 1
    return {"bytes": 2 * moved * case["page"] * token * case["layers"] + 2 * table, "flops": 0}


def _exact_attend(s):
    off, parents, lens = s.row_off.tolist(), s.parent.tolist(), s.lens.tolist()
    H, dh, Hkv = s.q.shape[1], s.q.shape[2], s.k.shape[2]
    outs, lses = [], []
    for b in range(len(off) - 1):
        n, length = off[b + 1] - off[b], lens[b]
        above, depth = [], []
        for i in range(n):
            p = parents[off[b] + i]
            line = {i} if p == -1 else (above[p] | {i} if 0 <= p < i and above[p] else set())
            above.append(line)
            depth.append(len(line) - 1)
        see = torch.zeros((n, length + n), dtype=torch.bool)
        for i in range(n):
            if above[i]:
                see[i, :length] = True
                if s.window > 0:
                    see[i, s.prefix:max(s.prefix, min(length, length + depth[i] - s.window + 1))] = False
                for j in above[i]:
                    see[i, length + j] = s.window == 0 or depth[i] - depth[j] < s.window
        see = see.cuda()
        pages = s.table[b, :-(-length // s.page)].long()
        k, v = (torch.cat([pool[0][pages].permute(1, 0, 2, 3).flatten(1, 2)[:, :length], x[off[b]:off[b + 1]].transpose(0, 1)], 1).double()
                for pool, x in ((s.k, s.k_new), (s.v, s.v_new)))
        q = s.q[off[b]:off[b + 1]].double()
        out, lse = torch.zeros((n, H, dh), dtype=torch.float64), torch.zeros((n, H), dtype=torch.float64)
        for h in range(H):
            z = (q[:, h] @ k[h // (H // Hkv)].T / math.sqrt(dh)).masked_fill(~see, float("-inf"))
            lse[:, h] = torch.logsumexp(z, 1).cpu()
            out[:, h] = (torch.nan_to_num(torch.softmax(z, 1)) @ v[h // (H // Hkv)]).cpu()
        outs.append(out)
        lses.append(lse)
    return torch.cat(outs), torch.cat(lses)


def exact(case, seed):
    """In 64 bits.  The page cases only move values: nothing there is computed."""
    if case["do"] not in ("attend", "score"):
        return None
    s = prepare(case, seed)
    if case["do"] == "attend":
        return _exact_attend(s)
    at = torch.arange(case["rows"], device="cuda")
    logprob, entropy, rank, ids, tops = [], [], [], [], []
    for part in at.split(256):
        z = torch.log_softmax(s.logits[part].double(), 1)
        mine = z[torch.arange(len(part), device="cuda"), s.tokens[part].long()]
        logprob.append(mine)
        entropy.append(-(z.exp() * z.masked_fill(torch.isinf(z), 0.0)).sum(1))
        x = s.logits[part].double()
        rank.append((x > x[torch.arange(len(part), device="cuda"), s.tokens[part].long()][:, None]).sum(1))
        order = x.sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
        ids.append(order)
        tops.append(z.gather(1, order))
    return torch.cat(logprob), torch.cat(entropy), torch.cat(rank).int(), torch.cat(ids).int(), torch.cat(tops)
