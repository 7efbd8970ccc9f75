"""Scores of logits rows whose unusual values stand where a row starts and ends: in front of the first and behind the last whole
vector of 16 bytes."""
import pytest

import test_gpu_tree_ops as T

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

if torch.cuda.is_available():
    from paper_2511_15618_b200 import logprobs


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [2049, 2061, 50001])
@pytest.mark.parametrize("top", [0, 1, 2, 20])
@pytest.mark.parametrize("where", [0, 1, -1, -2])
def test_one_value_far_above_the_rest_at_an_end_of_the_row(dtype, vocab, top, where):
    """Eight rows that start at every offset from a vector; the reference of the sums has to be the row's maximum."""
    torch.manual_seed(vocab + top)
    x = torch.randn((8, vocab + 9), device="cuda").to(dtype)[:, 1:1 + vocab]
    x[:, where] += 300
    t = torch.randint(vocab, (8,), device="cuda", dtype=torch.int32)
    t[::2] = where % vocab
    got = logprobs(x, t, top=top)
    T.check_scores(x, t, top, got)
    assert got[0][::2].abs().max() < 1e-30 and got[1].abs().max() < 1e-30      # all of the probability (the rest: e^-290)
