"""Trees of candidates through the whole model (fm_verify_tree, fm_accept_tree) against the oracle: every node's logits against a
chain pass over its path, the accepted path, and the state it leaves (drafts and chain passes that follow)."""
import numpy as np
import pytest

import fm_synth as S
import tree_reference as R
from test_gpu_parity import TOY, TOY_MARGIN, TOY_TOL, _dev, _setup

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def _np(x):
    return x.detach().cpu().numpy()


def _chain(cfg, seq, tokens):
    """The oracle's logits and predictions along a chain that starts with the pending token."""
    o, logits, margins = seq.verify(list(tokens) + [0] * (cfg.draft_len + 1 - len(tokens)))
    return o, logits, margins


def _tree_of(cfg, seq, rng, n):
    """Parents, tokens, and per node the oracle's prediction, logits and margin (None where no row is fed)."""
    parents, tokens, rows = [-1], [seq.main], []
    fed = min(cfg.draft_len + 1, seq.t_end - (seq.L - 1))
    for i in range(n):
        if i > 0:
            p = i - 1 if rng.random() < 0.5 else int(rng.integers(i))
            if rng.random() < 0.08:
                p = int(rng.choice([-1, -2, i, i + 3]))                    # no earlier node: out of use
            parents.append(p)
            good = 0 <= p < i and rows[p] is not None
            tokens.append(rows[p][0] if good and rng.random() < 0.65 else int(rng.integers(cfg.n_bins)))
        path = sorted(R.ancestors(parents)[i])
        if not path or path[0] != 0 or len(path) > fed:                   # (another root is none of this tree)
            rows.append(None)
            continue
        o, logits, margins = _chain(cfg, seq, [tokens[j] for j in path])
        rows.append((o[len(path) - 1], logits[len(path) - 1], margins[len(path) - 1]))
    return parents, tokens, rows


def _run(cfg, batch, faces, passes, seed, nodes=None, prompts_of=None):
    from oracle.hourglass import OracleSeq
    rng = np.random.default_rng(seed)
    w, conds, prompts = _setup(cfg, batch=batch)
    if prompts_of is not None:
        prompts = prompts_of(prompts)
    dev = _dev(cfg, w)
    seqs = [OracleSeq(cfg, w)]
    seqs += [OracleSeq(cfg, seqs[0].w) for _ in range(batch - 1)]
    for b, s in enumerate(seqs):
        s.prefill(conds[b], prompts[b], max_faces=faces[b])
    dev.prefill(np.stack(conds), prompts)
    dev.set_max_faces(faces)
    took = []
    for step in range(passes):
        if all(s.done for s in seqs):
            break
        if step % 3 == 2:                                                  # a chain pass in between: it reads what the trees left
            drafts = [s.draft() for s in seqs]
            cand, dl, _ = dev.draft(want_logits=True)
            for b, s in enumerate(seqs):
                if not s.done:
                    assert np.abs(_np(dl)[b] - drafts[b][1]).max() <= TOY_TOL
            cands = [d[0] for d in drafts]
            want = [s.verify(c) for s, c in zip(seqs, cands)]
            o, lg, _ = dev.verify(np.asarray(cands, dtype=np.int32), want_logits=True)
            for b, s in enumerate(seqs):
                assert s.rows == 0 or np.abs(_np(lg)[b, :s.rows] - want[b][1][:s.rows]).max() <= TOY_TOL
            n, em, kv = dev.accept(force_tok=np.asarray([x[0] for x in want], dtype=np.int32))
            for b, s in enumerate(seqs):
                a, e, k = s.accept()
                assert (int(n[b]), list(_np(em)[b]), tuple(_np(kv)[b])) == (a, e, k)
            continue
        N = nodes or int(rng.integers(1, cfg.draft_len + 2))
        tok, par, pred = (np.full((batch, N), v, dtype=np.int32) for v in (0, -2, -1))
        trees = []
        for b, s in enumerate(seqs):
            t = None if s.done else _tree_of(cfg, s, rng, N)
            trees.append(t)
            if t is not None:
                par[b], tok[b] = t[0], t[1]
                pred[b] = [r[0] if r is not None else -1 for r in t[2]]
        got, logits, _ = dev.verify_tree(tok, par, want_logits=True)
        got, logits = _np(got), _np(logits)
        again, _, _ = dev.verify_tree(tok, par)
        assert np.array_equal(_np(again), got)
        for b, t in enumerate(trees):
            for i in range(N):
                r = t[2][i] if t is not None else None
                if r is None:
                    assert got[b, i] == -1 and not logits[b, i].any()
                    continue
                assert np.abs(logits[b, i] - r[1]).max() <= TOY_TOL, (step, b, i)
                assert got[b, i] == r[0] or r[2] <= TOY_MARGIN
        path, n_acc, em, kv = (_np(x) for x in dev.accept_tree(force_pred=pred))
        for b, (s, t) in enumerate(zip(seqs, trees)):
            if t is None:
                assert n_acc[b] == 0 and (path[b] == -1).all()
                continue
            live = [p if r is not None else -2 for p, r in zip(t[0], t[2])]
            want, _ = R.accept(t[1], live, pred[b].tolist())
            tokens = [t[1][i] for i in want]
            if cfg.eos in tokens:
                want, tokens = want[:tokens.index(cfg.eos) + 1], tokens[:tokens.index(cfg.eos) + 1]
            assert path[b].tolist() == want + [-1] * (N - len(want)) and n_acc[b] == len(want)
            assert em[b].tolist() == tokens + [-1] * (N - len(want))
            _chain(cfg, s, tokens)
            a, _, k = s.accept(force_len=len(want))
            assert a == len(want) and tuple(kv[b]) == k
            took.append(a)
    assert dev.device_status() == 0
    assert max(took) > 2
    return took


@pytest.mark.parametrize("D", [3, 9, 12, 27])
@pytest.mark.parametrize("kv", [2, 1])
def test_trees_of_all_lengths(D, kv):
    cfg = S.toy_config(**TOY, draft_len=D, n_kv_heads=kv, layers=(1, 2, 2, 1, 2), max_batch=2, prompt_faces=(1, 1), gen_faces=8)
    cfg = cfg.with_(max_tokens=1 + 9 * 10 + D + 2)
    _run(cfg, 2, [8, 5], 9, D + kv, prompts_of=lambda p: [p[0], p[1] + p[0]])


def test_windows_that_wrap_around():
    cfg = S.toy_config(**TOY, draft_len=9, layers=(2, 1, 2, 2, 1), window=(11, 5, 2), n_kv_heads=1, allow_eos=1, max_batch=3, gen_faces=9,
                       max_tokens=1 + 9 * 10 + 9 + 2)
    _run(cfg, 3, [9, 9, 4], 30, 5)


def test_a_long_cache_and_a_window_of_whole_chunks():
    cfg = S.toy_config(**TOY, draft_len=9, window=(150, 70, 0), layers=(1, 1, 1, 1, 1), max_batch=2, prompt_faces=(60, 60), gen_faces=8)
    cfg = cfg.with_(max_tokens=1 + 9 * 72 + 9 + 2, prompt_subdiv=2)
    _run(cfg, 2, [8, 8], 8, 7, prompts_of=lambda p: [p[0], p[1][:9 * 31]])


def test_heads_of_128_and_full_draft_modules():
    cfg = S.toy_config(**{**TOY, "head_dim": 128, "d_model": 256, "d_ff": 512}, draft_len=9, draft_heads="full", hf_ff=192, layers=(1, 2, 1, 1, 2), max_batch=2,
                       prompt_faces=(1, 1), gen_faces=8, max_tokens=1 + 9 * 10 + 9 + 2)
    _run(cfg, 2, [8, 6], 8, 9)


def test_the_tiny_model_and_calls_out_of_order():
    from paper_2511_15618_b200 import FmError
    cfg = S.get_config("tiny", gen_faces=4)
    w, conds, prompts = _setup(cfg, batch=1)
    dev = _dev(cfg, w)
    dev.batch = 1
    with pytest.raises(FmError) as e:
        dev.verify_tree(np.zeros((1, 2)), np.zeros((1, 2)))
    assert e.value.code == -2
    dev.prefill(np.stack(conds), prompts)
    with pytest.raises(FmError) as e:
        dev.accept_tree()
    assert e.value.code == -2
    with pytest.raises(FmError) as e:
        dev.verify_tree(np.zeros((1, cfg.draft_len + 2)), np.full((1, cfg.draft_len + 2), -1))
    assert e.value.code == -3
    cand, _, _ = dev.draft()
    main = int(cand[0, 0])
    dev.verify_tree([[main, 1, 2, 3]], [[-1, 0, 0, 1]])
    with pytest.raises(FmError) as e:
        dev.accept()
    assert e.value.code == -2
    path, n, em, kv = dev.accept_tree()
    assert int(n[0]) >= 1 and int(em[0, 0]) == main and int(kv[0, 0]) == 1 + int(n[0])
    dev.verify_tree([[(main + 1) % cfg.n_bins]], [[-1]])                   # not the pending token
    assert dev.device_status() == -1


def test_alternatives_of_the_draft_heads_make_a_tree():
    """The run of the calls together: drafts, their top alternatives by logprobs, a tree of them, verified and accepted, until the end;
    the tokens are those of plain decoding wherever the oracle's margin says so."""
    from oracle.hourglass import OracleSeq
    D = 9
    cfg = S.toy_config(**TOY, draft_len=D, layers=(1, 1, 2, 1, 1), max_batch=1, prompt_faces=(1, 1), gen_faces=4, max_tokens=1 + 9 * 8 + D + 2)
    w, conds, prompts = _setup(cfg, batch=1)
    dev = _dev(cfg, w)
    s = OracleSeq(cfg, w)
    s.prefill(conds[0], prompts[0], max_faces=4)
    dev.prefill(np.stack(conds), prompts)
    dev.set_max_faces([4])
    out = []
    while len(out) < 36:
        cand, ids, lp, entropy = dev.draft_alternatives(2)
        first, second = ids[0, :, 0].tolist(), ids[0, :, 1].tolist()
        assert first == cand[0, 1:].tolist() and (lp[0, :, 0] >= lp[0, :, 1]).all() and (entropy >= 0).all()
        # a chain of the five first choices, and the second choice of the first four positions beside it
        tokens = [int(cand[0, 0])] + first[:5] + second[:4]
        parents = [-1, 0, 1, 2, 3, 4, 0, 1, 2, 3]
        pred, _, mg = dev.verify_tree([tokens], [parents])
        path, n, em, kv = dev.accept_tree()
        out += em[0, :int(n[0])].tolist()
    assert len(out) == 36 and dev.device_status() == 0
    # the oracle along the emitted tokens: each is its prediction, or all but tied
    for t in out:
        if s.main != t:
            assert s_margin <= TOY_MARGIN
        s.main = t
        _, _, margins = s.verify([t] + [0] * D)
        s_margin = margins[0]
        s.accept(force_len=1)
