"""kv_append_paged_mxfp8 against the definition of the format and of the append, bit for bit, and with nothing else touched."""
import numpy as np
import pytest
import torch

from mx_util import quantise
from paged_util import DEV, DTYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


def pools(pages, H, page, D, layout):
    """Codes and scales, K's and V's, full of a mark."""
    shape = (pages, H, page) if layout == "head" else (pages, page, H)
    made = [torch.full(shape + (n,), 0x5a, dtype=torch.uint8, device=DEV) for n in (D, D, D // 32, D // 32)]
    return [t.transpose(1, 2) if layout == "token" else t for t in made]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("H,D,page", [(2, 128, 16), (8, 64, 64), (3, 32, 32), (1, 96, 16), (5, 160, 16), (16, 128, 128)])
def test_against_the_definition(lotts, H, D, page, layout, dtype):
    print("mxfp8 append", H, D, page, layout, dtype, flush=True)
    g = torch.Generator().manual_seed(H + D)
    new, length = [1, 4, 0, 37, 3, 2], [1, page, 5, 37 + page, 2, 500]   # the fifth branch's first new token lies in front of its beginning; the last one's pages are missing
    starts = np.cumsum([0] + new)
    T, columns = int(starts[-1]) + 1, max(-(-n // page) for n in length[:5]) + 1   # one row behind the last branch's
    table = torch.full((6, columns), -1, dtype=torch.int32)
    ids = iter(torch.randperm(30, generator=g).tolist())
    for b in range(5):
        for c in range(-(-length[b] // page)):
            table[b, c] = next(ids)
    dt = DTYPES[dtype]
    qkv = (torch.randn(T, 2 * H + 3, D, generator=g) * torch.exp(2 * torch.randn(T, 2 * H + 3, 1, generator=g))).to(dt)
    qkv[3, 3:, 5] = float("inf")
    qkv[8, 3:, 31] = float("nan")
    qkv[9, 3:] = 0
    dev = qkv.to(DEV)
    Kc, Vc, Ks, Vs = pools(31, H, page, D, layout)
    want = [t.cpu().numpy().copy() for t in (Kc, Vc, Ks, Vs)]
    for half, (codes, scales) in enumerate(((want[0], want[2]), (want[1], want[3]))):
        c, s = quantise(qkv[:, 3 + half * H:3 + (half + 1) * H].float(), "mxfp8")
        for b in range(6):
            for i in range(new[b]):
                pos = length[b] - new[b] + i
                entry = int(table[b, pos // page]) if 0 <= pos < columns * page else -1
                if pos >= 0 and entry >= 0:
                    codes[entry, :, pos % page], scales[entry, :, pos % page] = c[starts[b] + i], s[starts[b] + i]
    f8, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    lotts.kv_append_paged_mxfp8(dev[:, 3:3 + H], dev[:, 3 + H:], Kc.view(f8), Vc.view(f8), Ks.view(e8), Vs.view(e8), table.to(DEV),
                                torch.tensor(length, dtype=torch.int32, device=DEV), torch.tensor(starts, dtype=torch.int32, device=DEV))
    for got, w in zip((Kc, Vc, Ks, Vs), want):
        assert np.array_equal(got.cpu().numpy(), w)


@pytest.mark.parametrize("B", [1, 64, 65, 300])
def test_many_branches(lotts, B):
    """More than 64 branches are searched in two steps; without q_start every branch has as many tokens."""
    H, D, page, n = 2, 64, 16, 3
    g = torch.Generator().manual_seed(B)
    new = torch.randn(B * n, H, D, generator=g).bfloat16()
    length = [n + (b * 37) % 60 for b in range(B)]
    table = torch.arange(B * 4, dtype=torch.int32).reshape(B, 4)
    made = []
    for start in (None, torch.arange(0, B * n + 1, n, dtype=torch.int32, device=DEV)):
        Kc, Vc, Ks, Vs = pools(B * 4, H, page, D, "head")
        rows = new.to(DEV)
        lotts.kv_append_paged_mxfp8(rows if start is not None else rows.view(B, n, H, D), rows if start is not None else rows.view(B, n, H, D), Kc, Vc, Ks, Vs,
                                    table.to(DEV), torch.tensor(length, dtype=torch.int32, device=DEV), start)
        made.append((Kc, Vc, Ks, Vs))
        c, s = quantise(new.float(), "mxfp8")
        codes, scales = np.full(Kc.shape, 0x5a, np.uint8), np.full(Ks.shape, 0x5a, np.uint8)
        for t in range(B * n):
            pos = length[t // n] - n + t % n
            codes[table[t // n, pos // page], :, pos % page], scales[table[t // n, pos // page], :, pos % page] = c[t], s[t]
        for got, w in zip((Kc, Vc, Ks, Vs), (codes, codes, scales, scales)):
            assert np.array_equal(got.cpu().numpy(), w)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_exponent(lotts, dtype):
    """Rows of every size, ties, subnormal numbers, zeros of both signs, the largest numbers."""
    g = np.random.default_rng(3)
    rows = [np.ldexp(np.concatenate([g.integers(-896, 897, 60) / 2, [448, -448, 0.0, -0.0]]), p) for p in range(-158, 119)]
    rows += [np.full(64, 3.3e38), np.where(np.arange(64) % 2, -3.3895e38, 1e38), np.full(64, -1e-45), np.zeros(64), -np.zeros(64)]
    x = torch.from_numpy(np.array(rows)).to(DTYPES[dtype])
    T = x.shape[0]
    Kc, Vc, Ks, Vs = pools(-(-T // 16), 1, 16, 64, "head")
    rows = x[:, None].to(DEV)
    lotts.kv_append_paged_mxfp8(rows, rows, Kc, Vc, Ks, Vs, torch.arange(-(-T // 16), dtype=torch.int32, device=DEV)[None], torch.tensor([T], dtype=torch.int32, device=DEV),
                                torch.tensor([0, T], dtype=torch.int32, device=DEV))
    c, s = quantise(x.float(), "mxfp8")
    for codes, scales in ((Kc, Ks), (Vc, Vs)):
        assert np.array_equal(codes.reshape(-1, 64)[:T].cpu().numpy(), c) and np.array_equal(scales.reshape(-1, 2)[:T].cpu().numpy(), s)
        assert (codes.reshape(-1, 64)[T:] == 0x5a).all()


def test_first_rows_that_do_not_ascend_and_lengths_that_no_table_holds(lotts):
    """Whatever the device data say, nothing outside the pages that the table names is written to."""
    H, D, page = 2, 64, 16
    rows = torch.randn(40, H, D, device=DEV).bfloat16()
    table = torch.arange(12, dtype=torch.int32, device=DEV).reshape(3, 4) + 1
    for starts, length in (([0, 40, 2, 4], [64, 64, 64]), ([5, 3, 1, 0], [9, 9, 9]), ([0, 2 ** 31 - 1, -2 ** 31, 7], [60, 5, 1]), ([0, 10, 20, 40], [2 ** 31 - 1, -5, 70])):
        Kc, Vc, Ks, Vs = pools(14, H, page, D, "head")
        lotts.kv_append_paged_mxfp8(rows, rows, Kc, Vc, Ks, Vs, table, torch.tensor(length, dtype=torch.int32, device=DEV),
                                    torch.tensor(starts, dtype=torch.int32, device=DEV))
        torch.cuda.synchronize()
        for t in (Kc, Vc, Ks, Vs):
            assert (t[0] == 0x5a).all() and (t[13] == 0x5a).all()
