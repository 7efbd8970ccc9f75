"""What a context reports of the launches of a tree pass: fm_launch_count, and the attention launches between fm_profile_begin and
fm_profile_end."""
import numpy as np
import pytest

import fm_synth as S
from test_gpu_parity import TOY, _dev, _setup

pytestmark = pytest.mark.gpu
pytest.importorskip("torch")

LAYERS = (2, 1, 3, 1, 1)


def context(tokens):
    cfg = S.toy_config(**TOY, draft_len=9, layers=LAYERS, max_batch=1, prompt_faces=(1, 1), gen_faces=4, max_tokens=tokens)
    w, conds, prompts = _setup(cfg, batch=1)
    dev = _dev(cfg, w)
    dev.prefill(np.stack(conds), prompts)
    main = int(dev.draft()[0][0, 0])
    return dev, [[main, 1, 2, 3]], [[-1, 0, 0, 1]]


def test_launches_of_a_tree_pass():
    """Caches of up to 768 positions are no more than eight chunks: no tile is cut, and none is merged.  Coordinates beyond that take a
    merge a layer, vertices (a third as many) do not."""
    counts = []
    for tokens in (200, 1200):
        dev, tok, par = context(tokens)
        dev.verify_tree(tok, par)
        before = dev.launch_count()
        dev.verify_tree(tok, par)
        counts.append(dev.launch_count() - before)
        before = dev.launch_count()
        dev.accept_tree()
        assert dev.launch_count() - before == 2
    assert counts[1] - counts[0] == LAYERS[0] + LAYERS[4]
    # five launches a layer at the most, two downwards and two upwards, tokens, maps, the logits' and the choice
    assert counts[0] >= 5 * sum(LAYERS) and counts[0] <= 5 * sum(LAYERS) + 14


def test_a_profile_has_the_attention_of_a_tree_pass():
    dev, tok, par = context(1200)
    dev.verify_tree(tok, par)
    dev.profile_begin()
    dev.verify_tree(tok, par)
    p = dev.profile_end()
    assert p.attn_launches == sum(LAYERS) and p.attn_ms > 0
