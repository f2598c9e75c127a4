"""skinny_gemm_mxfp4 against the product of the values that the weights stand for, in 64 bits."""
import math

import numpy as np
import pytest
import torch

from mx_util import pack, quantise, values
from paged_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


class Product:
    def __init__(self, M, N, K, seed=0, std=0.5):
        g = torch.Generator().manual_seed(seed)
        self.M, self.N, self.K = M, N, K
        W = torch.randn(N, K, generator=g) * K ** -0.5 * torch.exp(torch.randn(N, K // 32, generator=g)).repeat_interleave(32, 1)
        self.c, self.s = quantise(W, "mxfp4")
        self.x = (torch.randn(M, K, generator=g) * std).bfloat16()
        self.X, self.codes, self.scales = self.x.to(DEV), torch.from_numpy(pack(self.c)).to(DEV), torch.from_numpy(self.s).to(DEV)

    def reference(self):
        """Y in 64 bits and how far a kernel may be from it: the products of 8 and 2 bits are exact, their fp32 sums have at most one rounding or cut-off (a
        step, 2^-23) a product and one a partial sum of up to 64 shares of K, and the result is rounded to bf16 once (half a step, 2^-8)."""
        w = torch.from_numpy(values(self.c, self.s, "mxfp4"))
        Y = self.x.double() @ w.t()
        off = (self.K + 64) * 2.0 ** -23 * (self.x.double().abs() @ w.abs().t())
        return Y, off + 2.0 ** -8 * (Y.abs() + off)

    def check(self, got):
        Y, tol = self.reference()
        worst = ((got.cpu().double() - Y).abs() - tol).max().item()
        assert worst <= 0, worst   # (NaN is no number below 0)


SIZES = [(1, 1, 32), (1, 2560, 2048), (2, 33, 64), (5, 31, 96), (16, 64, 160), (17, 1003, 1056), (31, 40, 2080), (32, 256, 2048), (33, 300, 512), (64, 7168, 512),
         (65, 96, 5120), (100, 1, 1056), (128, 513, 992), (129, 130, 4096), (192, 257, 1120), (255, 700, 352), (256, 512, 1056), (256, 31, 32), (3, 20011, 64), (1, 7, 28672),
         (40, 5120, 288), (200, 2000, 1088)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_against_64_bits(lotts, M, N, K):
    print("mxfp4 product", M, N, K, flush=True)
    p = Product(M, N, K, seed=M + N + K)
    p.check(lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales))


@pytest.mark.parametrize("seed", range(24))
def test_sizes_at_random(lotts, seed):
    g = np.random.default_rng(seed)
    M, N, K = (int(round(math.exp(g.uniform(0, math.log(h))))) for h in (256, 6000, 160))
    print("mxfp4 product", M, N, 32 * K, flush=True)
    p = Product(M, N, 32 * K, seed=seed)
    p.check(lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales.view(torch.float8_e8m0fnu)))


@pytest.mark.parametrize("M,N,K", [(5, 100, 96), (64, 300, 2048), (200, 77, 1056), (1, 2560, 2048)])
def test_rows_that_lie_apart(lotts, M, N, K):
    """Views of larger buffers, an output of odd pitch that begins anywhere: nothing beside its rows is touched."""
    print("mxfp4 product, strides", M, N, K, flush=True)
    p = Product(M, N, K, seed=N)
    X = torch.full((M + 1, K + 24), math.nan, dtype=torch.bfloat16, device=DEV)
    codes = torch.full((N + 1, K // 2 + 48), 0x77, dtype=torch.uint8, device=DEV)
    scales = torch.full((N + 1, K // 32 + 5), 255, dtype=torch.uint8, device=DEV)
    X, codes, scales = X[:M, 8:8 + K], codes[:N, 16:16 + K // 2], scales[:N, 3:3 + K // 32]
    X.copy_(p.X), codes.copy_(p.codes), scales.copy_(p.scales)
    big = torch.full((M + 2, N + 5), 7.0, dtype=torch.bfloat16, device=DEV)
    out = lotts.skinny_gemm_mxfp4(X, codes, scales, out=big[1:M + 1, 3:3 + N])
    p.check(out)
    assert torch.equal(out, lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales))
    big[1:M + 1, 3:3 + N] = 7.0
    assert (big == 7.0).all()


@pytest.mark.parametrize("M,N,K", [(3, 70, 96), (40, 600, 1056), (64, 2560, 2048), (130, 64, 512)])
def test_what_is_no_number_stays_where_it_is(lotts, M, N, K):
    """A block of NaN in the last, odd place of K or in a neighbouring row; an infinity in a token."""
    p = Product(M, N, K, seed=K)
    clean = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
    rows = sorted({0, N // 2, N - 1})
    for i, n in enumerate(rows):
        p.scales[n, [0, K // 32 - 1, K // 64][i % 3]] = 255
    m = M // 2
    p.X[m, K - 1] = math.inf
    out = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
    off = torch.zeros((M, N), dtype=torch.bool, device=DEV)
    off[:, rows] = True
    assert torch.isnan(out[off]).all()
    off[m] = True
    assert torch.equal(out[~off], clean[~off]) and not torch.isfinite(out[m]).any()


def test_large_and_small_scales(lotts):
    """Powers of two in the weights' scales and in the tokens move the result by as much, exactly."""
    p = Product(9, 70, 512, seed=5)
    base = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
    for up in (-60, 60):
        s = (p.scales.to(torch.int32) + up).to(torch.uint8)
        assert torch.equal(lotts.skinny_gemm_mxfp4(p.X, p.codes, s).double(), base.double() * 2.0 ** up)
        assert torch.equal(lotts.skinny_gemm_mxfp4((p.X.double() * 2.0 ** -up).bfloat16(), p.codes, s), base)


def test_the_product_of_the_dequantised_weights(lotts):
    """The same weights in bf16 through skinny_gemm: the same product up to the order of the sums."""
    p = Product(60, 1000, 2048, seed=3)
    p.check(lotts.skinny_gemm(p.X, lotts.mxfp4_dequantize(p.codes, p.scales)))
    p.check(lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales))


@pytest.mark.parametrize("M,N,K", [(4, 1000, 1056), (64, 5120, 5120), (200, 640, 2048)])
def test_replays_streams_and_workspaces(lotts, M, N, K):
    """The same bits from a graph's replays, from another stream, with a workspace that holds anything, and call after call."""
    p = Product(M, N, K, seed=1)
    one = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
    need = lotts.load().skinny_gemm_mxfp4_workspace_bytes(M, N, K)
    ws = torch.randint(0, 255, (need,), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(one)
    call = lambda: lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales, out=out, workspace=ws)
    call()
    assert torch.equal(out, one)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(3):
        p.X.copy_((torch.randn(M, K, generator=torch.Generator().manual_seed(seed)) * 0.5).bfloat16())
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
        assert torch.equal(out, eager)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [torch.zeros_like(one) for _ in range(4)]
    torch.cuda.synchronize()
    for o in outs[:2]:
        lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales, out=o, stream=side)
    for o in outs[2:]:
        lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales, out=o)
    torch.cuda.synchronize()
    assert all(torch.equal(o, eager) for o in outs)


def test_weights_beyond_4_gib(lotts):
    """Rows behind 2^32 bytes of the codes."""
    N, K = 70000, 2048
    pitch = 1 << 16
    codes = torch.empty((N, pitch), dtype=torch.uint8, device=DEV)[:, :K // 2]
    p = Product(5, 300, K, seed=2)
    scales = torch.full((N, K // 32), 127, dtype=torch.uint8, device=DEV)
    codes.zero_()
    codes[-300:], scales[-300:] = p.codes, p.scales
    out = lotts.skinny_gemm_mxfp4(p.X, codes, scales)
    p.check(out[:, -300:])
    assert (out[:, :-300] == 0).all()


# Sizes at which each of the ways to cut the work is taken, with K's last chunk whole and not, K in one piece and in several; tokens and rows that fill no tile.
FORMS = [(20, 20000, 1056), (20, 20003, 512), (1, 40, 11040), (1, 40, 8192), (32, 9000, 1056), (1, 9001, 2048), (1, 1024, 11040), (3, 40, 16384),
         (33, 20000, 1056), (33, 20001, 512), (33, 40, 5152), (40, 41, 4096), (33, 9000, 2080), (64, 5000, 2048), (33, 5000, 2080), (63, 40, 16384),
         (70, 20000, 256), (70, 20001, 288), (96, 20000, 512), (70, 40, 5152), (70, 43, 4096), (100, 20000, 160), (100, 20000, 256), (100, 20000, 288),
         (128, 9000, 512), (100, 40, 5152), (127, 40, 5120), (130, 20000, 160), (131, 20002, 256), (130, 40, 11040), (191, 300, 8192), (256, 20000, 64),
         (200, 20000, 256), (200, 40, 11040), (201, 40, 9600), (256, 5120, 5120), (31, 55301, 1056), (31, 55300, 1280), (64, 55301, 1056), (64, 55297, 1280),
         (96, 55299, 1056), (96, 55300, 1280), (128, 55301, 1056), (128, 55300, 1280), (255, 55301, 1056), (255, 55300, 1280)]


class OnDevice:
    """Any codes, scales over a few powers of two; the reference is a product in 64 bits of what these stand for."""

    def __init__(self, M, N, K, ldx=None, ld_codes=None, ld_scales=None):
        g = torch.Generator(device=DEV).manual_seed(M + N + K)
        rows = lambda n, k, ld, dtype: torch.empty(n * (ld or k), dtype=dtype, device=DEV).view(n, ld or k)[:, :k]
        self.X, self.codes, self.scales = rows(M, K, ldx, torch.bfloat16), rows(N, K // 2, ld_codes, torch.uint8), rows(N, K // 32, ld_scales, torch.uint8)
        self.X.copy_(torch.randn(M, K, generator=g, device=DEV))
        self.codes.copy_(torch.randint(0, 256, self.codes.shape, generator=g, device=DEV, dtype=torch.uint8))
        self.scales.copy_(torch.randint(118, 124, self.scales.shape, generator=g, device=DEV, dtype=torch.uint8))

    def check(self, lotts, got):
        x, w = self.X.double(), lotts.mxfp4_dequantize(self.codes, self.scales, dtype=torch.float32).double()
        Y = x @ w.t()
        off = (x.shape[1] + 64) * 2.0 ** -23 * (x.abs() @ w.abs().t())
        assert ((got.double() - Y).abs() <= off + 2.0 ** -8 * (Y.abs() + off)).all()


@pytest.mark.parametrize("M,N,K", FORMS)
def test_every_cut(lotts, M, N, K):
    print("mxfp4 product", M, N, K, flush=True)
    p = OnDevice(M, N, K)
    out = torch.full((M, N + 3), 7.0, dtype=torch.bfloat16, device=DEV)
    p.check(lotts, lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales, out=out[:, :N]))
    assert (out[:, N:] == 7).all()


@pytest.mark.parametrize("M,N,K", [(256, 600, 16384), (100, 600, 16384), (20, 300, 16384), (3, 60, 512)])
def test_the_widest_pitches(lotts, M, N, K):
    """Rows of codes and scales 16 MiB apart, tokens 8 MiB: the last row of a workgroup lies 2^30 bytes and more behind its first."""
    print("mxfp4 product, widest pitches", M, N, K, flush=True)
    p = OnDevice(M, N, K, 1 << 22, 1 << 24, 1 << 24)
    p.check(lotts, lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales))


@pytest.mark.parametrize("M,N,K", [(5, 300, 96), (20, 20000, 1056), (1, 1024, 11040), (33, 40, 5152), (64, 9001, 2080), (70, 40, 5152), (100, 20000, 288), (130, 40, 11040),
                                   (200, 20000, 288), (256, 600, 16384)])
def test_what_lies_behind_rows_and_what_is_no_number(lotts, M, N, K):
    """NaN between the rows and behind the last one reaches nothing; a token's NaN reaches that token's row, a weight's that weight's column."""
    print("mxfp4 product, NaN", M, N, K, flush=True)
    p = OnDevice(M + 1, N + 1, K, K + 64, K // 2 + 32, K // 32 + 4)
    whole = lambda t, ld: t.as_strided((t.shape[0], ld), (ld, 1))
    X, codes, scales = p.X[:M].clone(), p.codes[:N].clone(), p.scales[:N].clone()
    whole(p.X, K + 64).fill_(math.nan)
    whole(p.scales, K // 32 + 4).fill_(255)
    p.X, p.codes, p.scales = p.X[:M].copy_(X), p.codes[:N].copy_(codes), p.scales[:N].copy_(scales)
    clean = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
    p.check(lotts, clean)
    m, n = M // 2, N // 3
    p.X[m, K - 1], p.scales[n, 0] = math.nan, 255
    got = lotts.skinny_gemm_mxfp4(p.X, p.codes, p.scales)
    bad = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    bad[m], bad[:, n] = True, True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], clean[~bad])
