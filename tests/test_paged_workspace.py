"""The paged attention's workspace query on the host: a buffer for a larger call serves the smaller ones."""
import ctypes

import pytest

import test_paged_abi
from test_paged_abi import lib  # noqa: F401  (a fixture)


@pytest.mark.parametrize("Hq,Hkv,D", [(16, 2, 128), (40, 8, 128), (8, 8, 64), (1, 1, 64), (5, 1, 128)])
def test_more_branches_and_more_new_tokens_never_ask_for_less(lib, Hq, Hkv, D):
    def ask(B, most):
        d = test_paged_abi.desc(B=B, T=B * most, max_new=most, Hq=Hq, Hkv=Hkv, D=D)
        return lib.verify_attention_paged_workspace_bytes(ctypes.byref(d))
    branches, mosts = [1, 2, 16, 63, 64, 65, 255, 256, 257, 511, 512, 513, 4096], list(range(1, 75))
    need = [[ask(B, m) for m in mosts if B * m * Hq < 1 << 24] for B in branches]
    for i, row in enumerate(need):
        assert all(n > 0 for n in row) and row == sorted(row), branches[i]
        if i:
            assert all(a <= b for a, b in zip(need[i - 1], row)), branches[i]
