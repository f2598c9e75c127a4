"""Where a matrix has one row, nothing is at the pitch: a token behind a long context, a row of a larger matrix.  Error paths only: the last check of a call answers."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ONE = ctypes.c_void_p(4096)   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(os.path.join(ROOT, "paper_2505_19634_amd", "liblotts.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2505_19634_amd import binding
    return binding.load()


def product(lib, M, N, K, ldx, lc, ls):
    few = lib.skinny_gemm_mxfp4_workspace_bytes(M, N, K) - 1
    return lib.skinny_gemm_mxfp4(M, N, K, ONE, ldx, ONE, lc, ONE, ls, ONE, N, ONE, few, None)


def test_the_product_takes_any_pitch_of_one_row(lib):
    assert product(lib, 1, 40, 5120, 5120, 2560, 160) == -4
    for ldx in (4096 * 5120, 5121, 1 << 40, 2 ** 63 - 1):
        assert product(lib, 1, 40, 5120, ldx, 2560, 160) == -4, ldx
        assert product(lib, 2, 40, 5120, ldx, 2560, 160) == -2, ldx
    for pitch in (1 << 30, 2561, 2 ** 63 - 1):
        assert product(lib, 5, 1, 5120, 5120, pitch, pitch) == -4, pitch
        assert product(lib, 5, 2, 5120, 5120, pitch, 160) == -2, pitch
    assert product(lib, 5, 2, 5120, 5120, 2560, 1 << 30) == -2
    # a row is as long as it is
    assert product(lib, 1, 40, 5120, 5119, 2560, 160) == -2 and product(lib, 5, 1, 5120, 5120, 2559, 160) == -2 and product(lib, 5, 1, 5120, 5120, 2560, 159) == -2
