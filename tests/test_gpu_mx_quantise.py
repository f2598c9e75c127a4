"""mxfp4_quantize and mxfp4_dequantize against the definition, bit for bit: codes with their signs, scales, values."""
import numpy as np
import pytest
import torch

from mx_util import KINDS, pack, quantise, unpack, values
from paged_util import DEV, DTYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


def check(lotts, W, **outs):
    codes, scales = lotts.mxfp4_quantize(W.to(DEV) if not W.is_cuda else W, **outs)
    want, s = quantise(W.cpu().float(), "mxfp4")
    assert codes.dtype == torch.uint8 and scales.element_size() == 1
    assert np.array_equal(scales.view(torch.uint8).cpu().numpy(), s)
    assert np.array_equal(codes.cpu().numpy(), pack(want))
    v = values(want, s, "mxfp4")
    for dtype in (torch.bfloat16, torch.float32):
        got = lotts.mxfp4_dequantize(codes, scales, dtype=dtype)
        assert got.dtype == dtype and np.array_equal(got.double().cpu().numpy(), v, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,K", [(1, 32), (3, 64), (7, 96), (65, 32), (1003, 1056), (2, 28672), (300, 2048)])
def test_matrices(lotts, N, K, dtype):
    print("mxfp4", N, K, dtype, flush=True)
    g = torch.Generator().manual_seed(N + K)
    check(lotts, (torch.randn(N, K, generator=g) * torch.exp(torch.randn(N, 1, generator=g) * 3)).to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_exponent(lotts, dtype):
    """Rows of every size, halves of elements among them, so that there are ties; subnormal numbers; zeros of both signs; the largest numbers."""
    rows = []
    elements = KINDS["mxfp4"][0]
    ties = np.concatenate([(elements[1:] + elements[:-1]) / 2, elements, [5.9, 0.24, 0.26, 2.49, 2.51]])
    for p in range(-149, 126):
        x = np.concatenate([ties, -ties])[:32] if p % 2 else -np.concatenate([ties, -ties])[-32:]
        x = np.resize(x, 32).copy()
        x[7] = 6.0
        rows.append(np.ldexp(x, p))
    rows += [np.zeros(32), -np.zeros(32), np.full(32, 3.3e38), np.where(np.arange(32) % 2, -3.3895e38, 1e38), np.full(32, 1e-45), np.full(32, -1e-40)]
    check(lotts, torch.from_numpy(np.array(rows)).to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_is_no_number(lotts, dtype):
    W = torch.randn(6, 96)
    W[0, 3], W[1, 40], W[2, 95], W[3, 0], W[3, 64] = float("inf"), float("nan"), -float("inf"), float("nan"), float("inf")
    check(lotts, W.to(DTYPES[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_lie_apart(lotts, dtype):
    """Strided matrix, codes, scales and values; nothing between the rows is touched."""
    N, K = 9, 160
    big = torch.randn(N, K + 64).to(DTYPES[dtype]).to(DEV)
    W = big[:, 32:32 + K]
    codes = torch.full((N, 128), 0xee, dtype=torch.uint8, device=DEV)
    scales = torch.full((N, 11), 0xee, dtype=torch.uint8, device=DEV)
    check(lotts, W, codes=codes[:, 16:16 + K // 2], scales=scales[:, 3:3 + K // 32])
    assert (codes[:, :16] == 0xee).all() and (codes[:, 16 + K // 2:] == 0xee).all()
    assert (scales[:, :3] == 0xee).all() and (scales[:, 3 + K // 32:] == 0xee).all()
    out = torch.full((N, K + 32), 7.0, dtype=DTYPES[dtype], device=DEV)
    lotts.mxfp4_dequantize(codes[:, 16:16 + K // 2], scales[:, 3:3 + K // 32], out=out[:, 16:16 + K])
    assert torch.equal(out[:, 16:16 + K].float(), lotts.mxfp4_dequantize(codes[:, 16:16 + K // 2].contiguous(), scales[:, 3:3 + K // 32].contiguous()).float())
    assert (out[:, :16] == 7.0).all() and (out[:, 16 + K:] == 7.0).all()


def test_every_code_with_every_scale(lotts):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    want = values(unpack(codes), scales, "mxfp4")
    for dtype in (torch.bfloat16, torch.float32):
        got = lotts.mxfp4_dequantize(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), dtype=dtype)
        assert np.array_equal(got.double().cpu().numpy(), np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want), equal_nan=True)


def test_a_stream_of_its_own_and_a_graph(lotts):
    W = torch.randn(130, 1056, device=DEV)
    codes, scales = lotts.mxfp4_quantize(W)
    out = lotts.mxfp4_dequantize(codes, scales)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    c2, s2 = torch.zeros_like(codes), torch.zeros_like(scales.view(torch.uint8))
    torch.cuda.synchronize()
    lotts.mxfp4_quantize(W, codes=c2, scales=s2, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(c2, codes) and torch.equal(s2, scales.view(torch.uint8))
    graph, o2 = torch.cuda.CUDAGraph(), torch.zeros_like(out)
    with torch.cuda.graph(graph):
        lotts.mxfp4_quantize(W, codes=c2, scales=s2)
        lotts.mxfp4_dequantize(c2, s2, out=o2)
    for seed in range(4):
        W.copy_(torch.randn(130, 1056, generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        codes, scales = lotts.mxfp4_quantize(W)
        assert torch.equal(c2, codes) and torch.equal(o2, lotts.mxfp4_dequantize(codes, scales))
