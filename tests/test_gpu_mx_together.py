"""The microscaled calls as a decoder makes them: a projection of MXFP4 weights whose K and V go into an MXFP8 cache that forks and grows, and the attention over
it, eager and captured, against the same steps in 64 bits on the values that weights and cache stand for."""
import math

import numpy as np
import pytest
import torch

import paged_util as P
from mx_util import pack, quantise, values

DEV = P.DEV
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_a_generation(lotts, captured):
    B, Hq, Hkv, D, page, columns, pages, hidden = 5, 8, 2, 64, 16, 9, 60, 160
    g = torch.Generator().manual_seed(5)
    N, T = (Hq + 2 * Hkv) * D, 37
    W = (torch.randn(N, hidden, generator=g) * hidden ** -0.5).bfloat16()
    codes, scales = lotts.mxfp4_quantize(W.to(DEV))
    c4, s4 = quantise(W.float(), "mxfp4")
    assert np.array_equal(codes.cpu().numpy(), pack(c4))
    w = torch.from_numpy(values(c4, s4, "mxfp4"))
    pool = torch.full((2, pages, Hkv, page, D), 0x7f, dtype=torch.uint8, device=DEV)          # K and V; NaN
    scale_pool = torch.full((2, pages, Hkv, page, D // 32), 255, dtype=torch.uint8, device=DEV)
    table = torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
    refs, kv_len = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    new_t, q_start = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    X, qkv = torch.zeros(T, hidden, dtype=torch.bfloat16, device=DEV), torch.zeros(T, N, dtype=torch.bfloat16, device=DEV)
    heads = qkv.view(T, Hq + 2 * Hkv, D)
    out, lse = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, Hq, device=DEV)
    copies, missing = torch.zeros(B, 2, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws, gemm_ws, attn_ws = (torch.zeros(n << 20, dtype=torch.uint8, device=DEV) for n in (1, 64, 256))

    def enqueue():
        lotts.skinny_gemm_mxfp4(X, codes, scales, out=qkv, workspace=gemm_ws)
        lotts.kv_pages_reserve(table, refs, kv_len, new_t, page, copies=copies, missing=missing, workspace=ws)
        lotts.kv_pages_copy(pool, copies)
        lotts.kv_pages_copy(scale_pool, copies)
        lotts.kv_append_paged_mxfp8(heads[:, Hq:Hq + Hkv], heads[:, Hq + Hkv:], pool[0], pool[1], scale_pool[0], scale_pool[1], table, kv_len, q_start)
        lotts.verify_attention_paged_mxfp8(heads[:, :Hq], pool[0], pool[1], scale_pool[0], scale_pool[1], table, kv_len, q_start, out=out, lse=lse, workspace=attn_ws)

    graph = None
    if captured:
        enqueue()   # with no new tokens: nothing changes
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            enqueue()
    tokens = [[] for _ in range(B)]   # (k, v) of every token of a branch: what the cache holds of them

    def step(new):
        x = torch.randn(T, hidden, generator=g).bfloat16()
        X.copy_(x)
        new_t.copy_(torch.tensor(new, dtype=torch.int32))
        q_start.copy_(torch.tensor([sum(new[:b]) for b in range(B + 1)], dtype=torch.int32))
        graph.replay() if captured else enqueue()
        torch.cuda.synchronize()
        assert missing.item() == 0
        n = sum(new)
        y = qkv.cpu().double()
        exact = x.double() @ w.t()
        off = (hidden + 64) * 2.0 ** -23 * (x.double().abs() @ w.abs().t())
        assert ((y - exact).abs() <= off + 2.0 ** -8 * (exact.abs() + off)).all()
        rows = y.view(T, Hq + 2 * Hkv, D)
        held = values(*quantise(rows[:, Hq:], "mxfp8"), "mxfp8")
        ref = P.Cache(new, [len(t) + m for t, m in zip(tokens, new)], Hq, Hkv, D, page, device="cpu")
        ref.q = qkv.cpu().view(T, Hq + 2 * Hkv, D)[:n, :Hq]
        for b in range(B):
            for i in range(new[b]):
                row = torch.from_numpy(held[ref.starts[b] + i])
                tokens[b].append((row[:Hkv], row[Hkv:]))
            for j, mine in enumerate((ref.k, ref.v)):
                mine[b] = torch.stack([t[j] for t in tokens[b]]) if tokens[b] else torch.zeros(0, Hkv, D, dtype=torch.float64)
        P.check(ref, out[:n], lse[:n])
        assert kv_len.tolist() == [len(t) for t in tokens]

    step([T, 0, 0, 0, 0])
    step([11, 0, 0, 0, 0])
    lotts.kv_pages_fork(table, refs, kv_len, torch.zeros(B, dtype=torch.int32, device=DEV))
    tokens = [list(tokens[0]) for _ in range(B)]
    for turn in range(5):
        step([4, 1, 3, 2, 4])
        for b in range(B):   # the last token is taken back
            tokens[b].pop()
        kv_len.sub_(1)
        if turn == 3:
            lotts.kv_pages_free(table, refs, kv_len, page)
            moves, counts = lotts.kv_pages_compact(table, refs)
            lotts.kv_pages_copy(pool, moves, count=counts)
            lotts.kv_pages_copy(scale_pool, moves, count=counts)


def test_a_projection_larger_than_the_step(lotts):
    """One decoder layer of 3B shape from weights to attention's output, against 64 bits from the same quantised weights: the QKV product feeds the cache, the
    attention its output product."""
    B, n, Hq, Hkv, D, page, hidden, L = 8, 4, 16, 2, 128, 64, 2048, 500
    g = torch.Generator().manual_seed(6)
    new, length = [n] * B, [L - 13 * b for b in range(B)]
    from mx_util import MxCache
    c = MxCache(new, length, Hq, Hkv, D, page, seed=6)
    x = torch.randn(B * n, hidden, generator=g).bfloat16()
    Wqkv, Wo = ((torch.randn(r, k, generator=g) * k ** -0.5).bfloat16() for r, k in (((Hq + 2 * Hkv) * D, hidden), (hidden, Hq * D)))
    qkv4, o4 = lotts.mxfp4_quantize(Wqkv.to(DEV)), lotts.mxfp4_quantize(Wo.to(DEV))
    heads = lotts.skinny_gemm_mxfp4(x.to(DEV), *qkv4).view(B, n, Hq + 2 * Hkv, D)
    lotts.kv_append_paged_mxfp8(heads[:, :, Hq:Hq + Hkv], heads[:, :, Hq + Hkv:], *c.cache, c.table, c.kv_len)
    attn = lotts.verify_attention_paged_mxfp8(heads[:, :, :Hq], *c.cache, c.table, c.kv_len)
    Y = lotts.skinny_gemm_mxfp4(attn.view(B * n, Hq * D), *o4)
    held = torch.from_numpy(values(*quantise(heads[:, :, Hq:].cpu().float(), "mxfp8"), "mxfp8"))
    for b in range(B):
        c.k[b][-n:], c.v[b][-n:] = held[b, :, :Hkv], held[b, :, Hkv:]
    c.q = heads[:, :, :Hq].reshape(B * n, Hq, D).cpu()
    P.check(c, attn.view(B * n, Hq, D))
    a = attn.view(B * n, Hq * D).cpu().double()
    w = torch.from_numpy(values(*quantise(Wo.float(), "mxfp4"), "mxfp4"))
    exact, off = a @ w.t(), (Hq * D + 64) * 2.0 ** -23 * (a.abs() @ w.abs().t())
    assert ((Y.cpu().double() - exact).abs() <= off + 2.0 ** -8 * (exact.abs() + off)).all()
    assert math.isfinite(float(Y.float().abs().max()))


def test_the_whole_stack_step_of_the_latency_model(lotts):
    """Two layers of a tiny decoder with MXFP4 weights and a paged MXFP8 cache, a prefix that ends inside a page: the last layer's products and attention against 64
    bits from what went into them, and replays of the captured step against the eager one, bit for bit."""
    from mx_util import unpack
    from paper_2505_19634_amd import latency_model as lm
    shape = lm.ModelShape("tiny decoder", 2, 512, 8, 2, 64, 1024, 4096)
    B, R, prefix, private = 4, 3, 150, 70
    fm = lm.MicroscaledModel(shape, prefix, private, B, R - 1)
    fm.enqueue()
    torch.cuda.synchronize()
    results = (fm.qkv, fm.attn, fm.gu, fm.o, fm.zt, fm.accept_len, fm.next_token) + fm.layers[0]["cache"] + fm.layers[1]["cache"]
    raw = lambda t: t.view(torch.uint8) if t.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu) else t
    want = [raw(t).clone() for t in results]
    last, w64 = fm.layers[1], lambda pair: torch.from_numpy(values(unpack(pair[0].cpu().numpy()), raw(pair[1]).cpu().numpy(), "mxfp4"))

    def product(x, pair, got):
        x, w = x.cpu().double(), w64(pair)
        exact, off = x @ w.t(), (x.shape[1] + 64) * 2.0 ** -23 * (x.abs() @ w.abs().t())
        assert ((got.cpu().double() - exact).abs() <= off + 2.0 ** -8 * (exact.abs() + off)).all()
    a = fm.attn.view(B * R, -1)
    o = torch.empty_like(fm.o)
    lotts.skinny_gemm_mxfp4(a, *last["o"], out=o, workspace=fm.ws_gemm)
    product(a, last["o"], o)
    product(o, last["gate_up"], fm.gu)
    product(fm.gu[:, :shape.mlp], last["down"], fm.o)
    # the cache: the pages of the prefix are shared, the rest is each branch's own, the last rows are the step's
    L, page = prefix + private + R, fm.PAGE
    table = fm.table.cpu()
    assert (table[:, :prefix // page] == table[0, :prefix // page]).all() and len(set(table[:, prefix // page:].flatten().tolist())) == table[:, prefix // page:].numel()
    c = P.Cache([R] * B, [L] * B, shape.Hq, shape.Hkv, shape.D, page, device="cpu")
    held = [torch.from_numpy(values(raw(x).cpu().numpy(), raw(y).cpu().numpy(), "mxfp8")) for x, y in zip(last["cache"][:2], last["cache"][2:])]
    c.k, c.v = ([h[table[b].long()].transpose(1, 2).reshape(-1, shape.Hkv, shape.D)[:L] for b in range(B)] for h in held)
    heads = fm.qkv.cpu().view(B * R, -1, shape.D)
    new = torch.from_numpy(values(*quantise(heads[:, shape.Hq:].float(), "mxfp8"), "mxfp8")).view(B, R, 2, shape.Hkv, shape.D)
    for b in range(B):
        assert torch.equal(c.k[b][-R:], new[b, :, 0]) and torch.equal(c.v[b][-R:], new[b, :, 1])
    c.q = heads[:, :shape.Hq]
    P.check(c, fm.attn.view(B * R, shape.Hq, shape.D))
    for t in results[:5]:
        t.zero_()
    assert fm.step_ms(reps=3) > 0.0
    for turn in range(2):
        for got, was in zip(results, want):
            assert torch.equal(raw(got), was)
        fm.attn.zero_()
        fm.graph.replay()
        torch.cuda.synchronize()
    with pytest.raises(ValueError):
        lm.MicroscaledModel(shape, 64, 64, 100, 2)
