"""The microscaled calls on one row, wherever its matrix would have the next one: the last token of a long context, a row of a matrix of odd pitch."""
import pytest
import torch

from mx_sums import rounded, whole_product
from paged_util import DEV, DTYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


@pytest.mark.parametrize("N,K", [(300, 5120), (20003, 1312), (40, 27648)])
def test_the_last_token_of_a_context(lotts, N, K):
    """hidden[:, -1] of one branch: a pitch of the whole context."""
    print("mxfp4 product, last token", N, K, flush=True)
    X, codes, scales, w = whole_product(1, N, K, device=DEV)
    hidden = torch.full((1, (1 << 22) // K + 2, K), float("nan"), dtype=torch.bfloat16, device=DEV)
    hidden[:, -1] = X
    last = hidden[:, -1]
    assert last.stride(0) > 1 << 22
    assert torch.equal(lotts.skinny_gemm_mxfp4(last, codes, scales), rounded(X.double() @ w.t()))


@pytest.mark.parametrize("M,K", [(1, 1312), (5, 5120), (64, 11040), (200, 512)])
def test_one_row_of_weights(lotts, M, K):
    print("mxfp4 product, one row of weights", M, K, flush=True)
    X, codes, scales, w = whole_product(M, 1, K, device=DEV)
    far = lambda t, pitch: t.reshape(-1).as_strided(t.shape, (pitch, 1))   # (the pitch of a row that has no neighbour)
    want = rounded(X.double() @ w.t())
    for pitch in (K // 2 + 1, 1 << 30):
        assert torch.equal(lotts.skinny_gemm_mxfp4(X, far(codes, pitch), far(scales, pitch)), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_of_a_matrix_of_odd_pitch(lotts, dtype):
    K = 1056
    W = torch.randn(3, K + 1, generator=torch.Generator().manual_seed(1)).to(DTYPES[dtype]).to(DEV)[:1, :K]
    codes, scales = (torch.zeros(2, n + 1, dtype=torch.uint8, device=DEV)[:1, :n] for n in (K // 2, K // 32))
    lotts.mxfp4_quantize(W, codes=codes, scales=scales)
    want_codes, want_scales = lotts.mxfp4_quantize(W.clone(memory_format=torch.contiguous_format))
    assert torch.equal(codes, want_codes) and torch.equal(scales, want_scales.view(torch.uint8))
    out = torch.full((2, K + 1), 7.0, dtype=DTYPES[dtype], device=DEV)
    lotts.mxfp4_dequantize(codes, scales, out=out[:1, :K])
    assert torch.equal(out[:1, :K], lotts.mxfp4_dequantize(want_codes, want_scales, dtype=DTYPES[dtype]))
    assert (out[0, K:] == 7.0).all() and (out[1] == 7.0).all()
