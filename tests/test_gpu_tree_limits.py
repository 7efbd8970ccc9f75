"""Limits that change between the pass over a tree and its acceptance: no more is accepted than of a chain."""
import numpy as np
import pytest

import fm_synth as S
from test_gpu_parity import TOY, _dev, _setup

pytestmark = pytest.mark.gpu
pytest.importorskip("torch")


@pytest.mark.parametrize("faces,most", [(8, 10), (2, 10), (1, 9), (0, 0)])
def test_a_limit_lowered_behind_the_pass(faces, most):
    D = 9
    cfg = S.toy_config(**TOY, draft_len=D, layers=(1, 1, 1, 1, 1), max_batch=1, prompt_faces=(1, 1), gen_faces=8, max_tokens=1 + 9 * 10 + D + 2)
    w, conds, prompts = _setup(cfg, batch=1)
    got = []
    for tree in (True, False):
        dev = _dev(cfg, w)
        dev.prefill(np.stack(conds), prompts)
        dev.set_max_faces([8])
        main = int(dev.draft()[0][0, 0])
        tokens = [main] + [(3 * i) % cfg.n_bins for i in range(D)]
        pred = np.asarray([tokens[1:] + [5]], dtype=np.int32)             # a chain that is confirmed to its end
        if tree:
            dev.verify_tree([tokens], [list(range(-1, D))])
        else:
            dev.verify(np.asarray([tokens], dtype=np.int32))
        dev.set_max_faces([faces])
        if tree:
            path, n, em, kv = dev.accept_tree(force_pred=pred)
            assert path[0].tolist() == list(range(most)) + [-1] * (D + 1 - most)
        else:
            n, em, kv = dev.accept(force_tok=pred)
        assert int(n[0]) == most and em[0].tolist() == tokens[:most] + [-1] * (D + 1 - most)
        assert dev.device_status() == 0
        # finished or not: what the next pass says
        cand, _, _ = dev.draft()
        dev.verify(cand)
        n2, _, kv2 = dev.accept()
        got.append((kv.tolist(), int(n2[0]) > 0))
    assert got[0] == got[1] and got[0][1] == (faces >= 2)
