"""fm_verify_tree and fm_accept_tree without a device: what they refuse."""
from paper_2511_15618_b200 import binding as B
from paper_2511_15618_b200.build import build


def test_no_context():
    build()
    assert B.fm_verify_tree(None, 1 << 20, 1 << 20, 2) == -1
    assert B.fm_accept_tree(None) == -1
