"""`PagedCache.check` and calls on other streams than the one that it is called on; errors of very large calls."""
import pytest

import test_gpu_tree_ops as T

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_an_error_of_a_call_that_still_waits_on_another_stream():
    c = T.PagedCache(1, 4, 4, 1, 64, 2, 2)
    seqs, grow = T.dev([0, 5]), T.dev([1, 1])                            # there is no sequence 5
    c.reserve(T.dev([0]), T.dev([1]))                                     # (the first launch of a kernel loads it, and may wait for the device)
    c.check()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)                                    # (0.1 s)
        c.reserve(seqs, grow)
    with pytest.raises(T.FmError) as e:
        c.check()
    assert e.value.code == -1
    c.check()


def test_entries_that_want_more_than_2_to_31_pages_in_all():
    """4096 entries of 2^19 pages each, in a pool of 64: they get none, and the small one behind them is served."""
    S, P = 4096, 2 ** 19
    c = T.PagedCache(1, 64, 1, 1, 8, S, P, dtype=torch.bfloat16)
    seqs = torch.arange(S, dtype=torch.int32, device="cuda")
    grow = torch.full((S,), P, dtype=torch.int32, device="cuda")
    grow[S - 1] = 3
    c.reserve(seqs, grow)
    with pytest.raises(T.FmError) as e:
        c.check()
    assert e.value.code == -3
    assert c.table[S - 1, :4].tolist() == [0, 1, 2, -1] and c.refs.tolist() == [1] * 3 + [0] * 61
    assert int((c.table != -1).sum()) == 3 and int(c.lens.abs().sum()) == 0
    c.reserve(seqs[:2], T.dev([60, 2]))                                   # as always: the first takes what there is
    with pytest.raises(T.FmError):
        c.check()
    assert c.refs.tolist() == [1] * 63 + [0] and c.table[0, :61].tolist() == list(range(3, 63)) + [-1]
