"""Scores of logits rows whose unusual values stand where a row starts and ends: in front of the first and behind the last whole
vector of 16 bytes."""
import math

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


def test_the_longest_row():
    """2^31 - 1 equal values: nothing can be collected by a bound, so the row is walked over once more, to its very end."""
    vocab = 2 ** 31 - 1
    x = torch.zeros((1, vocab), device="cuda", dtype=torch.bfloat16)
    lp, ent, rank, ids, tops = logprobs(x, T.dev([vocab - 1]), top=3)
    want = math.log(vocab)
    # a thread's sum of ones is exact (below 2^24); 5 additions in a warp and 15 of warps round, half a step of 2^-24 each; the
    # logarithm and what follows it four roundings of a value of that size
    tol = 24 * 2.0 ** -24 + 4 * 2.0 ** -24 * want
    assert rank.item() == 0 and ids[0].tolist() == [0, 1, 2]
    assert abs(lp.item() + want) <= tol and abs(ent.item() - want) <= tol and ((tops + want).abs() <= tol).all()
    x[0, vocab - 1] = 1.0
    lp, ent, rank, ids, tops = logprobs(x, T.dev([0]), top=3)
    assert rank.item() == 1 and ids[0].tolist() == [vocab - 1, 0, 1]
