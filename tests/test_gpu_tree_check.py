"""`PagedCache.check` and calls on other streams than the one that it is called on."""
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
