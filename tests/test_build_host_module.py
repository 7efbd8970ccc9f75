"""When the module of native functions for torch tensors is built again: not by the times of the files alone (no compiler runs here)."""
import os

import pytest

from paper_2511_15618_b200 import build as B


@pytest.fixture
def asked(monkeypatch):
    B.build()
    out = []
    monkeypatch.setattr(B, "_run", lambda cmd, what: out.append(what))
    return out


def test_nothing_is_built_twice(asked):
    B.build()
    assert asked == []
    from paper_2511_15618_b200 import trees
    assert trees._host().__doc__ == B._built_for()


@pytest.mark.parametrize("other", ["torch", "python"])
def test_another_torch_or_python(asked, monkeypatch, other):
    if other == "torch":
        monkeypatch.setattr(B.importlib.metadata, "version", lambda name: "2.99.0+cu130")
    else:
        monkeypatch.setattr(B.sysconfig, "get_config_var", lambda name: "cpython-399-x86_64-linux-gnu")
    B.build()
    assert asked == ["g++ failed building _trees.so"]


def test_a_module_cut_short_or_of_an_older_source(asked, monkeypatch, tmp_path):
    part = tmp_path / "_trees.so"
    part.write_bytes(open(B.HOST, "rb").read()[:1000])
    monkeypatch.setattr(B, "HOST", str(part))
    B.build()
    assert len(asked) == 1
    part.write_bytes(B._built_for().encode())
    B.build()
    assert len(asked) == 1
    os.utime(part, (0, 0))
    B.build()
    assert len(asked) == 2
