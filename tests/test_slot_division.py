"""Division of slots and rows by a constant, as the tree attention does it: the multiplier and shift of the built library, the product
in 64 bits and its halves in 32 as on the device."""
import ctypes as C

import numpy as np
import pytest

from paper_2511_15618_b200.build import build


class Div(C.Structure):
    _fields_ = [("mul", C.c_uint32), ("shift", C.c_int32), ("d", C.c_int32)]


@pytest.fixture(scope="module")
def div_by():
    f = C.CDLL(build())["_ZN2tr6div_byEi"]                 # tr::div_by(int)
    f.restype, f.argtypes = Div, [C.c_int32]
    return f


def quotient(v, n):
    """Div::operator(): n itself for d = 1, else the high word of the product, shifted."""
    if v.d == 1:
        return n
    return ((n.astype(np.uint64) * np.uint64(v.mul)) >> np.uint64(32)).astype(np.uint32) >> np.uint32(v.shift)


def test_quotients(div_by):
    rng = np.random.default_rng(1)
    small, large = range(1, 700), [1 << k for k in range(31)] + [(1 << k) - 1 for k in range(2, 32)] + [(1 << k) + 1 for k in range(2, 31)]
    for d in sorted(set(small) | set(large) | set(rng.integers(1, 2 ** 31, 300).tolist())):
        v = div_by(d)
        assert v.d == d and (d == 1 or 0 <= v.shift < 32)
        whole = np.minimum((np.arange(0, 400, dtype=np.int64) * max(1, 2 ** 31 // d // 399)) * d, 2 ** 31 - 1)
        n = np.concatenate([rng.integers(0, 2 ** 31, 400), np.arange(400), 2 ** 31 - 1 - np.arange(400), whole, np.maximum(whole - 1, 0)]).astype(np.int64)
        assert (quotient(v, n) == n // d).all(), d
