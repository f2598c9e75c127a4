"""verify_attention_paged_mxfp8 over every code with every scale byte: rows of one key, whose weight is 1, so that O is V's row as the kernel reads it, and the
score one element of K's.  bf16 rows read every value as a bf16 number (the nearest, ties to the even one; infinite from 2^128 on), fp32 rows as it is."""
import math

import numpy as np
import pytest
import torch

from mx_util import values
from paged_util import DEV, DTYPES

pytestmark = pytest.mark.gpu

# Query heads for the KV head: a narrow item's one row tile, its two row tiles, a wide item's rows.
HEADS = [2, 40, 72]


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


def rows_of(D, lo, hi, codes):
    """Rows that hold every one of `codes` under every scale byte from lo to hi, a scale a row: codes [rows][D], scales [rows][D / 32]."""
    each = np.resize(codes, -(-len(codes) // D) * D).reshape(-1, D).astype(np.uint8)
    s = np.repeat(np.arange(lo, hi + 1, dtype=np.uint8), len(each))
    return np.tile(each, (hi - lo + 1, 1)), np.repeat(s[:, None], D // 32, 1)


def read(codes, scales, dtype):
    """What a kernel reads of them."""
    v = torch.from_numpy(values(codes, scales, "mxfp8"))
    return v.float().to(DTYPES[dtype]).double()   # (fp32 holds every one below 2^128)


class OneKey:
    """Branch b has one token, in page b; what the branch does not hold is NaN.  The operand that is not given holds ones."""

    def __init__(self, B, D, K=None, V=None):
        def pages(row):
            c, s = np.full((B, 1, 16, D), 0x7f, np.uint8), np.full((B, 1, 16, D // 32), 255, np.uint8)
            c[:, 0, 0], s[:, 0, 0] = (0x38, 127) if row is None else row
            return torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV)
        (Kc, Ks), (Vc, Vs) = pages(K), pages(V)
        self.cache = Kc, Vc, Ks, Vs
        self.table = torch.arange(B, dtype=torch.int32, device=DEV)[:, None].contiguous()
        self.kv_len = torch.ones(B, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("new", [1, 3])
def test_values(lotts, new, heads, D, dtype):
    """With more new tokens than the branch has, the last one sees the key and the others nothing."""
    print("mxfp8 values", new, heads, D, dtype, flush=True)
    codes, scales = rows_of(D, 0, 255, np.arange(256))
    B = len(codes)
    want = read(codes, scales, dtype)[:, None, None].expand(B, 1, heads, D)
    c = OneKey(B, D, V=(codes, scales))
    Q = torch.randn(B, new, heads, D, generator=torch.Generator().manual_seed(D)).to(DTYPES[dtype]).to(DEV)
    for part in (slice(0, B), slice(0, B // 4), slice(B // 4, B // 2), slice(B // 2, B)):   # (in large calls two workgroups share a unit)
        got = lotts.verify_attention_paged_mxfp8(Q[part], *c.cache, c.table[part], c.kv_len[part]).cpu().double()
        assert (got[:, :-1] == 0).all()
        there = want[part].isfinite()
        assert torch.equal(got[:, -1:][there], want[part][there])
        assert not got[:, -1:][~there].isfinite().any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [h for h in HEADS if h != 2] + [32])
def test_scores(lotts, heads, D, dtype):
    """Head h's query is a power of two in column h + first and zero elsewhere: the score is an element of K times that power, which lse holds.  Scales up to
    246, under which every element is finite."""
    print("mxfp8 scores", heads, D, dtype, flush=True)
    codes, scales = rows_of(D, 0, 246, [c for c in range(256) if c & 0x7f != 0x7f])
    B = len(codes)
    c = OneKey(B, D, K=(codes, scales))
    up = torch.exp2(127.0 - torch.from_numpy(scales[:, 0]).double())
    k = read(codes, scales, dtype) * up[:, None]
    for first in range(0, D, heads):
        n = min(heads, D - first)
        Q = torch.zeros(B, 1, heads, D, dtype=torch.float64)
        Q[:, 0, torch.arange(n), first + torch.arange(n)] = up[:, None]
        _, lse = lotts.verify_attention_paged_mxfp8(Q.to(DTYPES[dtype]).to(DEV), *c.cache, c.table, c.kv_len, scale=1.0, return_lse=True)
        got, want = lse.cpu().double()[:, :n], k[:, first:first + n]
        # the score is exact; the scale, its factor log2 e, what takes that back and their products are off by half a step each
        assert ((got - want).abs() <= 8 * 2.0 ** -24 * want.abs()).all(), ((got - want).abs() - 8 * 2.0 ** -24 * want.abs()).max()
        assert (lse[:, n:] == 0).all()
