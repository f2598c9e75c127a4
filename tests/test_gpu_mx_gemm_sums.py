"""skinny_gemm_mxfp4 where the sums are exact in any order: equal to the product in 64 bits, rounded once, for long K and for every way to cut it."""
import pytest
import torch

from mx_sums import rounded, whole_product
from paged_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


# Long K in one to four groups of wavefronts and up to 24 splits, its last chunk whole and not, for every number of token tiles; short K straight from memory.
SIZES = [(1, 7, 28672), (1, 40, 27648), (3, 40, 16384), (5, 5120, 27648), (20, 1024, 27680), (20, 20003, 1312), (31, 55301, 1056), (1, 1024, 11040), (17, 9000, 1056),
         (33, 7, 27648), (40, 1024, 27680), (64, 5120, 27648), (40, 20000, 6912), (40, 9000, 2080), (64, 55301, 5120), (70, 40, 27648), (96, 5120, 27680), (70, 20001, 1056),
         (96, 55299, 1056), (128, 1024, 27648), (100, 9000, 11040), (128, 55301, 1056), (140, 300, 27680), (192, 5120, 27648), (130, 20000, 160), (200, 40, 27648),
         (256, 5120, 27648), (255, 55301, 1056), (256, 20000, 64), (129, 2048, 11008)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_the_sums_are_whole(lotts, M, N, K):
    print("mxfp4 product, exact sums", M, N, K, flush=True)
    X, codes, scales, w = whole_product(M, N, K, device=DEV)
    assert torch.equal(lotts.skinny_gemm_mxfp4(X, codes, scales), rounded(X.double() @ w.t()))
