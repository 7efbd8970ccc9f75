"""The rows that an attention call says it has: what is refused without a device."""
import pytest

import test_tree_refusals as T
from test_tree_refusals import lib                         # noqa: F401 (the built library)


@pytest.mark.parametrize("bad", [dict(n_rows=-1), dict(n_rows=0, fill=1), dict(n_rows=8, fill=4), dict(n_rows=8, fill=-1)])
def test_rows_and_fills(lib, bad):                         # noqa: F811
    assert lib.fm_tree_attention_bytes(T.cache(), T.args(n_rows=8, fill=3)) > 0
    assert lib.fm_tree_attention_bytes(T.cache(), T.args(n_rows=8)) > 0
    assert lib.fm_tree_attention_bytes(T.cache(), T.args(**bad)) == 0
    assert lib.fm_tree_attention(T.cache(), 0, T.args(**bad), T.P, 1 << 30, None) == T.INVALID


def test_rows_of_appends_and_acceptance(lib):              # noqa: F811
    p, c = T.pages(), T.cache()
    append = lambda n_rows: lib.fm_pages_append(p, c, bytes(T.T.FmNewRows(T.P, T.P, 0, 128, 64, n_rows)), T.P, T.P, None, 0, None, 0, 1, None)
    assert append(7) == 0 and append(0) == 0 and append(-1) == T.INVALID
    assert lib.fm_tree_accept_rows(T.P, T.P, T.P, T.P, -1, 2, T.P, 4, T.P, T.P, None) == T.INVALID
    assert lib.fm_tree_accept_rows(T.P, T.P, T.P, T.P, 8, 0, T.P, 4, T.P, T.P, None) == T.INVALID
    assert lib.fm_tree_accept_rows(T.P, None, T.P, T.P, 8, 2, T.P, 4, T.P, T.P, None) == T.INVALID
