"""The tree attention's large tiles on small inputs.  A pass takes them by what the caller says of its sizes: tables with room for
many positions, and trees that may have 256 nodes, make a pass of few positions a large one."""
import functools

import pytest

import test_gpu_tree_ops as T

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(autouse=True)
def large(monkeypatch):
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2511_15618_b200 import PagedCache
    filled, attention = T.filled, PagedCache.attention

    def roomy(rng, lens, Hkv, dh, page, dtype, max_pages=None, **kw):
        return filled(rng, lens, Hkv, dh, page, dtype, max_pages=max_pages or -(-200000 // page), **kw)

    @functools.wraps(attention)
    def many(self, layer, q, k_new, v_new, row_off, parent, **kw):
        if len(row_off) == 2 and kw.get("window"):                       # (a window bounds what a pass reads: 19 trees without nodes)
            row_off = torch.cat([row_off, row_off[-1:].expand(19)])
            kw["seqs"] = torch.zeros(20, dtype=torch.int32, device="cuda")
        return attention(self, layer, q, k_new, v_new, row_off, parent, **{**kw, "max_nodes": 256})

    monkeypatch.setattr(T, "filled", roomy)
    monkeypatch.setattr(PagedCache, "attention", many)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("heads,Hkv", [(2, 2), (4, 1), (7, 1), (24, 3)])
def test_types_and_heads(dtype, dh, heads, Hkv):
    T.run_case(31, [37, 0, 200, 1], [5, 3, 9, 1], heads, Hkv, dh, 16, dtype)


@pytest.mark.parametrize("length", [0, 1, 2, 63, 64, 65, 127, 128, 129, 500, 1023, 4100])
@pytest.mark.parametrize("nodes", [1, 4, 28])
def test_lengths(length, nodes):
    T.run_case(32, [length], [nodes], 4, 2, 64, 64, BF)
    T.run_case(33, [length, 77], [nodes, 2], 4, 4, 128, 24, HF)


@pytest.mark.parametrize("page", [1, 2, 3, 4, 6, 7, 8, 12, 16, 20, 24, 36, 40, 100, 256])
def test_page_sizes(page):
    T.run_case(34, [211, 90], [6, 11], 4, 2, 64, page, BF)
    T.run_case(34, [330, 90], [6, 11], 4, 2, 128, page, BF)


@pytest.mark.parametrize("nodes", [2, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 200, 256])
def test_tree_sizes(nodes):
    T.run_case(35, [70], [nodes], 2, 1, 64, 16, BF)
    T.run_case(36, [33, 130], [nodes, 1], 8, 1, 128, 16, BF)


@pytest.mark.parametrize("window", [1, 5, 64, 100, 250])
@pytest.mark.parametrize("prefix", [0, 1, 64, 130, 400])
def test_windows(window, prefix):
    T.run_case(37, [300, 129, 10] * 40, [20, 7, 1] * 40, 4, 2, 64, 16, BF, window=window, prefix=prefix)
    T.run_case(38, [300, 140] * 30, [40, 2] * 30, 4, 1, 128, 32, HF, window=window, prefix=prefix)


@pytest.mark.parametrize("heads,nodes", [(2, 6), (8, 40)])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_has_no_effect(dh, heads, nodes, what):
    T.test_what_a_row_does_not_see_has_no_effect(dh, heads, 1, nodes, what)


def test_bad_pages_are_refused_on_the_device():
    T.test_bad_pages_are_refused_on_the_device()


def test_the_same_call_gives_the_same_bits_and_replays():
    T.test_the_same_call_gives_the_same_bits_and_replays()
