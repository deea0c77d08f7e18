"""Refusals of the weight, eviction and tree calls that are checked on the host alone (no GPU needed)."""
import ctypes

import pytest

from paper_2412_12706_b200 import build as qp_build
from paper_2412_12706_b200 import qp
from tests.test_abi_weights import A, cache


@pytest.fixture(scope="module")
def lib():
    qp_build.build()
    return qp.lib()


@pytest.mark.parametrize("off", [1, 2, 3])
def test_pointers_that_are_not_aligned_to_their_type(lib, off):
    """Arrays of 32-bit numbers that the kernels read and write one by one: four bytes are enough, fewer are refused."""
    for name in ("weights", "kept", "kept_weights", "kept_pos"):
        p = dict(weights=A, kept=A, kept_weights=A, kept_pos=A)
        p[name] += off
        assert lib.qp_heavy_select(p["weights"], 1, 2, 256, 32, 64, 64, p["kept"], p["kept_weights"], p["kept_pos"], None) == 5, name
    c = cache(cap=80)
    assert lib.qp_evict_kv(A, A, ctypes.byref(c), None, A, A, 100, 8, A + off, None) == 5
    assert c.n_keep == 64                                                # nothing changed
