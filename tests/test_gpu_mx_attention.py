"""verify_attention_paged_mxfp8 against its definition in 64 bits on the values that the cache stands for: chunks, drafts and single tokens beside each other,
branches without new tokens or without any, pages of every size in either order, missing pages, rows that see nothing, NaN in every place that no branch
holds and in keys that only some rows see."""
import math

import pytest
import torch

from mx_util import MxCache
from paged_util import DEV, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


def attend(lotts, c, scale=0.0, max_new=None, workspace=None):
    out = torch.full((c.q.shape[0] + 2,) + c.q.shape[1:], 7.0, dtype=c.q.dtype, device=DEV)
    lse = torch.full((c.q.shape[0] + 2, c.Hq), 7.0, device=DEV)
    T = c.q.shape[0]
    # rows behind the last branch's: there, but nobody's
    Q = torch.cat([c.Q, torch.full((2,) + c.Q.shape[1:], float("nan"), dtype=c.Q.dtype, device=DEV)])
    lotts.verify_attention_paged_mxfp8(Q, *c.cache, c.table, c.kv_len, c.q_start, scale=scale, out=out, lse=lse, max_new=max_new, workspace=workspace)
    torch.cuda.synchronize()
    assert (out[T:] == 7.0).all() and (lse[T:] == 7.0).all()
    return out[:T], lse[:T]


MIXES = {  # (new tokens, all tokens) of the branches
    "one": [(1, 1)],
    "one_of_many": [(1, 777)],
    "drafts": [(4, 100), (4, 4), (4, 65), (4, 513)],
    "empty": [(0, 0), (3, 50), (0, 40), (2, 2), (0, 0)],
    "blind": [(5, 3), (40, 2), (2, 0), (3, 20)],            # more new tokens than the branch has: the first rows see nothing
    "mixed": [(1, 300), (133, 133), (2, 31), (64, 200), (1, 16), (32, 33)],
    "chunk": [(257, 700), (1, 1000)],
    "pages_end": [(1, 16), (1, 17), (2, 32), (3, 64), (1, 63), (5, 128), (1, 129)],
}
HEADS = [(16, 2, 128), (8, 8, 64), (5, 1, 128), (28, 4, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,page", [("head", 16), ("token", 64)])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("mix", sorted(MIXES))
def test_against_64_bits(lotts, mix, Hq, Hkv, D, layout, page, dtype):
    print("mxfp8 attention", mix, Hq, Hkv, D, layout, page, dtype, flush=True)
    new, length = zip(*MIXES[mix])
    c = MxCache(new, length, Hq, Hkv, D, page, dtype, layout, seed=len(mix) + Hq)
    check(c, *attend(lotts, c))
    if max(new) < sum(new):
        check(c, *attend(lotts, c, max_new=max(new)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("n,L", [(1, 2049), (3, 5000), (17, 1500), (70, 1111)])
def test_lengths(lotts, n, L, page, dtype):
    print("mxfp8 attention", n, L, page, dtype, flush=True)
    c = MxCache([n, 1], [L, L // 3], 4, 2, 64 if page == 32 else 128, page, dtype, seed=n)
    check(c, *attend(lotts, c, max_new=n))


@pytest.mark.parametrize("B", [63, 64, 65, 130, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_branches(lotts, B, dtype):
    print("mxfp8 attention", B, dtype, flush=True)
    new = [(b * 7) % 4 for b in range(B)]
    length = [n + (b * 37) % 90 for b, n in enumerate(new)]
    c = MxCache(new, length, 4, 2, 64, 16, dtype, seed=B)
    check(c, *attend(lotts, c, max_new=3))


@pytest.mark.parametrize("tiny", [3, 100, 400])
@pytest.mark.parametrize("chunk,L", [(90, 90), (150, 1000), (700, 3100)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_chunk_beside_tiny_branches(lotts, tiny, chunk, L, D):
    """The work's equal pieces may be as small as a tile of the chunk is long: every one of them has a part of it."""
    print("mxfp8 attention", tiny, chunk, L, D, flush=True)
    new = [1 + b % 2 for b in range(tiny // 2)] + [chunk] + [1] * (tiny - tiny // 2)
    length = [n + b % 3 for b, n in enumerate(new)]
    length[tiny // 2] = L
    c = MxCache(new, length, 4, 2 if tiny < 100 else 1, D, 16, seed=tiny + chunk)
    check(c, *attend(lotts, c, max_new=chunk))


@pytest.mark.parametrize("n,L,Hq,Hkv", [(300, 300, 16, 2), (1030, 1500, 8, 8), (513, 4000, 5, 1), (2039, 2039, 16, 2), (260, 9000, 2, 1)])
def test_prompts(lotts, n, L, Hq, Hkv):
    print("mxfp8 attention", n, L, Hq, Hkv, flush=True)
    c = MxCache([n], [L], Hq, Hkv, 128 if Hq != 5 else 64, 64, seed=n)
    check(c, *attend(lotts, c, max_new=n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_missing_pages(lotts, page, dtype):
    print("mxfp8 attention, missing pages", page, dtype, flush=True)
    holes = [(0, 0, -1), (0, 3, 0), (1, 1, -7), (2, 0, -1), (2, 1, 2 ** 30), (3, 5, -1), (3, 6, -1)]
    c = MxCache([2, 80, 3, 1], [4 * page + 5, 2 * page + 9, 2 * page, 9 * page], 8, 2, 128, page, dtype, holes=holes, seed=page)
    check(c, *attend(lotts, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_as_many_tokens_of_every_branch(lotts, dtype):
    """Without q_start, Q [B][n][Hq][D] a view of a projection's output, out one of a larger buffer; codes and scales as plain bytes."""
    B, n, Hq, Hkv, D = 6, 3, 10, 2, 64
    c = MxCache([n] * B, [40, 3, 129, 77, 64, 15], Hq, Hkv, D, 32, dtype, seed=3, types=(torch.uint8, torch.uint8))
    qkv = torch.full((B * n, Hq + 2 * Hkv, D), float("nan"), dtype=c.q.dtype, device=DEV)
    qkv[:, :Hq] = c.Q
    big = torch.full((B, n, Hq + 1, D), 7.0, dtype=c.q.dtype, device=DEV)
    out, lse = lotts.verify_attention_paged_mxfp8(qkv.view(B, n, Hq + 2 * Hkv, D)[:, :, :Hq], *c.cache, c.table, c.kv_len, out=big[:, :, :Hq], return_lse=True)
    assert out.shape == (B, n, Hq, D) and lse.shape == (B * n, Hq)
    check(c, out, lse)
    assert (big[:, :, Hq] == 7.0).all()
    flat = lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len)
    assert torch.equal(flat.view(B, n, Hq, D), out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_lie_apart(lotts, D, dtype):
    """Scale rows of three times their length, code rows further apart than they are long."""
    c = MxCache([4, 100, 1], [300, 160, 77], 8, 2, D, 16, dtype, seed=D)
    pages, Hkv, page = c.Kc.shape[:3]
    one = lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len, c.q_start)
    wide = [torch.full((pages, Hkv, page + 1, D + 48), 0x7f, dtype=torch.uint8, device=DEV)[:, :, :page, 16:16 + D] for _ in range(2)]
    odd = [torch.full((pages, Hkv, page, 3 * (D // 32)), 255, dtype=torch.uint8, device=DEV)[..., D // 32:2 * (D // 32)] for _ in range(2)]
    for t, s in zip(wide + odd, c.cache):
        t.copy_(s.view(torch.uint8))
    out = lotts.verify_attention_paged_mxfp8(c.Q, *wide, *odd, c.table, c.kv_len, c.q_start)
    assert torch.equal(out, one)
    check(c, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.03, 0.5])
def test_scale_and_wide_scores(lotts, scale, dtype):
    """Scores of some hundreds: nearly all weight on one key."""
    c = MxCache([3, 50], [300, 210], 4, 2, 128, 16, dtype, seed=8, std=3.0)
    check(c, *attend(lotts, c, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(1, 4), (20, 2), (300, 1)], ids=str)
def test_a_scale_that_leaves_nothing_of_the_scores(lotts, new, dtype):
    c = MxCache(new, [n + 700 for n in new], 8, 2, 128, 16, dtype, seed=8)
    for scale in (1e-38, 2e-39):
        check(c, *attend(lotts, c, scale=scale, max_new=max(new)), scale=scale)


def test_blocks_of_very_different_sizes(lotts):
    """K and V whose blocks lie far apart, as their scales allow: large values beside ones that nothing is left of."""
    c = MxCache([4, 90], [500, 300], 8, 2, 128, 16, seed=11)
    up = torch.tensor([0, -20, 4, -60], device=DEV)   # of the four blocks of a row
    for s, mine in ((c.Ks, c.k), (c.Vs, c.v)):
        b = s.view(torch.uint8)
        b.copy_(torch.where(b == 255, 255, b.to(torch.int32) + up).to(torch.uint8))
        for b_ in range(2):
            mine[b_] = mine[b_] * torch.exp2(up.cpu().double()).repeat_interleave(32)
    check(c, *attend(lotts, c))
    check(c, *attend(lotts, c, max_new=90))


def test_against_the_cache_in_bf16(lotts):
    """The values of the cache in bf16 pages through verify_attention_paged: the same attention."""
    c = MxCache([4, 70, 1], [700, 333, 64], 16, 2, 128, 16, seed=2)
    wide = lambda codes, scales: (codes.float() * scales.float().repeat_interleave(32, -1)).bfloat16()
    K, V = wide(c.Kc, c.Ks), wide(c.Vc, c.Vs)
    check(c, lotts.verify_attention_paged(c.Q, K, V, c.table, c.kv_len, c.q_start))
    check(c, *attend(lotts, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_beyond_4_gib(lotts, dtype):
    """Pages behind 2^32 bytes of the pool, and scales behind 2^32 bytes of theirs."""
    page, Hkv, D = 64, 8, 128
    pages = (5 << 30) // (Hkv * page * D)
    c = MxCache([3, 40], [300, 120], 16, Hkv, D, page, dtype, seed=4)
    far = torch.arange(c.Kc.shape[0], device=DEV) + (pages - c.Kc.shape[0])
    new = []
    for t, gap in zip(c.cache, (0, 0, 60, 60)):
        big = torch.empty((pages, Hkv, page, t.shape[3] + gap), dtype=torch.uint8, device=DEV)[..., :t.shape[3]]
        big.zero_()
        big[far] = t.view(torch.uint8)
        new.append(big)
    c.Kc, c.Vc, c.Ks, c.Vs = new
    c.table = torch.where(c.table >= 0, c.table + (pages - far.numel()), c.table)
    check(c, *attend(lotts, c))
    check(c, *attend(lotts, c, max_new=40))


def test_replays(lotts):
    """Captured once, replayed with other lengths, other pages and other numbers of new tokens."""
    first = MxCache([2, 30, 1], [100, 64, 257], 16, 2, 128, 16, seed=0, spare_pages=40, more_columns=30)
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(first.Q)
    lse = torch.zeros(first.q.shape[:2], device=DEV)
    call = lambda: lotts.verify_attention_paged_mxfp8(first.Q, *first.cache, first.table, first.kv_len, first.q_start, out=out, lse=lse, max_new=32, workspace=ws)
    call()
    torch.cuda.synchronize()
    check(first, out, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed, (new, length) in enumerate([((2, 30, 1), (100, 64, 257)), ((1, 0, 32), (500, 0, 90)), ((31, 1, 1), (31, 333, 16)), ((2, 30, 1), (5, 450, 3))]):
        other = MxCache(new, length, 16, 2, 128, 16, seed=seed + 50)
        for mine, its in zip(first.cache, other.cache):
            mine.view(torch.uint8)[:its.shape[0]] = its.view(torch.uint8)
        first.table.fill_(-1)
        first.table[:, :other.table.shape[1]] = other.table
        first.Q.copy_(other.Q)
        first.kv_len.copy_(other.kv_len)
        first.q_start.copy_(other.q_start)
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        check(other, out, lse)
        eager = torch.zeros_like(out)
        lotts.verify_attention_paged_mxfp8(first.Q, *first.cache, first.table, first.kv_len, first.q_start, out=eager, max_new=32, workspace=ws)
        assert torch.equal(eager, out)


def test_streams_with_workspaces_of_their_own(lotts):
    """Calls that overlap in time, one a stream, and then all of them on one stream with one workspace: the same bits."""
    cases = [MxCache(new, length, 16, 2, 128, 16, seed=i) for i, (new, length) in enumerate([((3, 1), (900, 4000)), ((300, 2), (700, 2500)), ((9, 9, 9), (100, 3000, 50))])]
    streams = [torch.cuda.Stream() for _ in cases]
    one = [lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len, c.q_start, max_new=max(c.new), return_lse=True) for c in cases]
    torch.cuda.synchronize()
    outs = [torch.zeros_like(c.Q) for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, st, o in zip(cases, streams, outs):
            lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len, c.q_start, max_new=max(c.new), out=o, stream=st)
    torch.cuda.synchronize()
    for c, (a, lse), b in zip(cases, one, outs):
        assert torch.equal(a, b)
        check(c, a, lse)


def test_a_workspace_that_an_unfinished_call_left(lotts):
    """Cells with an old tag and a count, anything in the partials: as good as zeros."""
    c = MxCache([4, 300], [3000, 1500], 16, 2, 128, 16, seed=1)
    clean = attend(lotts, c, max_new=300)
    ws = torch.randint(0, 2 ** 31, (64 << 20,), dtype=torch.int32, device=DEV)
    ws[:4096] = torch.tensor([(1 << 16) + 3, 0], dtype=torch.int32, device=DEV).repeat(2048)   # 64-bit cells: tag 1, three arrivals
    dirty = attend(lotts, c, max_new=300, workspace=ws.view(torch.uint8))
    for a, b in zip(clean, dirty):
        assert torch.equal(a, b)


def test_one_workspace_for_every_kind_of_call(lotts):
    """Calls that lay their partials out differently take turns with one buffer, which is as large as the largest asks for; all of them cut branches."""
    many = MxCache([1] * 260, [30] * 259 + [7000], 4, 2, 128, 16, seed=1)
    cases = [(many, 1), (MxCache([300, 1], [2500, 900], 8, 2, 64, 16, seed=2), 300), (MxCache([4, 2], [5000, 800], 8, 2, 128, 32, seed=3), 4),
             (MxCache([12], [3000], 8, 2, 128, 16, seed=4), 12), (MxCache([3, 1], [100, 60], 4, 2, 64, 16, "f32", seed=5), 3)]
    ws = torch.zeros(80 << 20, dtype=torch.uint8, device=DEV)
    first = [attend(lotts, c, max_new=n) for c, n in cases]
    for a, (c, _) in zip(first, cases):
        check(c, *a)
    for order in (range(5), (4, 3, 2, 1, 0), (1, 0, 3, 0, 2, 0, 4, 0)):
        for i in order:
            again = attend(lotts, cases[i][0], max_new=cases[i][1], workspace=ws)
            assert all(torch.equal(a, b) for a, b in zip(first[i], again)), i


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("most", [1, 5])
def test_more_items_than_twice_the_units(lotts, D, most):
    """One branch is much longer than the others and is cut many times, some are empty."""
    new = [(i * 7) % (most + 1) for i in range(270)]
    length = [n + (i * 37) % 150 for i, n in enumerate(new)]
    new[100], length[100] = most, 9000
    c = MxCache(new, length, 4, 2, D, 16, seed=D)
    check(c, *attend(lotts, c, max_new=most))


NANS = {
    "drafts": [(4, 100), (4, 4), (4, 65), (4, 513), (1, 40)],
    "two_row_tiles": [(16, 300), (9, 33), (12, 12)],
    "blind": [(5, 3), (40, 20), (3, 20), (70, 30)],
    "chunks": [(257, 700), (1, 1000), (60, 200), (300, 300)],
    "cut": [(6, 9000), (290, 4000)],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("by", ["code", "scale", "overflow"])
@pytest.mark.parametrize("Hq,Hkv,D,page,layout", [(16, 2, 128, 16, "head"), (4, 4, 64, 64, "token"), (8, 1, 64, 16, "head")])
@pytest.mark.parametrize("mix", sorted(NANS))
def test_nan_in_v_reaches_only_rows_that_see_the_key(lotts, mix, Hq, Hkv, D, page, layout, by, dtype):
    """A code that is NaN, a block whose scale makes it NaN, a code whose value no bf16 and no fp32 holds."""
    print("not finite", mix, Hq, Hkv, D, page, layout, by, dtype, flush=True)
    new, length = zip(*NANS[mix])
    c = MxCache(new, length, Hq, Hkv, D, page, dtype, layout, seed=len(mix) + D)
    g = torch.Generator().manual_seed(D + Hq)
    off = torch.zeros(c.q.shape, dtype=torch.bool)
    codes, scales = c.Vc.view(torch.uint8), c.Vs.view(torch.uint8)
    for b, (n, L) in enumerate(NANS[mix]):
        first = L - n
        keys = {L - 1, max(0, first + n // 2), max(0, first), max(0, first + 1) if n > 1 else L - 1} - ({max(0, first)} if b % 2 else set())
        for key in sorted(keys):
            h, block = int(torch.randint(0, Hkv, (1,), generator=g)), int(torch.randint(0, D // 32, (1,), generator=g))
            entry = int(c.table[b, key // page])
            if by == "code":
                at = torch.tensor([block * 32 + 3, block * 32 + 17])
                codes[entry, h, key % page, at.to(DEV)] = 0x7f
            else:
                at = torch.arange(block * 32, block * 32 + 32)
                scales[entry, h, key % page, block] = 255 if by == "scale" else 254
                if by == "overflow":
                    codes[entry, h, key % page, at.to(DEV)] = 0x7e
            c.v[b][key, h, at] = 0.0
            for i in range(max(0, key - first), n):
                rows = off[c.starts[b] + i, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)]
                rows[:, at] = True
    O, ref_lse, tol, tol_lse = c.reference()
    for max_new in {max(new), c.q.shape[0]}:
        out, lse = lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len, c.q_start, max_new=max_new, return_lse=True)
        got, l = out.cpu().double(), lse.cpu().double()
        assert not torch.isfinite(got[off]).any()
        worst = ((got - O).abs() - tol)[~off].max().item()
        assert worst <= 0, worst   # (NaN is no number below 0)
        seen = ~torch.isinf(ref_lse)
        assert ((l - ref_lse).abs() <= tol_lse)[seen].all() and torch.isinf(l[~seen]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_page_of_nothing_but_nan(lotts, dtype):
    """Every key of V is NaN: rows that see one are NaN, blind ones 0."""
    c = MxCache([5, 40, 3], [3, 30, 200], 8, 2, 128, 16, dtype, seed=3)
    c.Vs.view(torch.uint8).fill_(255)
    for max_new in (40, 48):
        out = lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len, c.q_start, max_new=max_new).cpu()
        blind = torch.zeros(48, dtype=torch.bool)
        blind[0:2] = blind[5:15] = True
        assert (out[blind] == 0).all() and torch.isnan(out[~blind]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_device_data_outside_the_contract(lotts, dtype):
    """Lengths that no table holds, first rows that do not ascend: nothing outside the outputs' rows changes, the other branches' rows are as without."""
    c = MxCache([3, 2, 1, 3, 40], [200, 30, 90, 64, 150], 8, 2, 64, 16, dtype, seed=3)
    T, (B, columns) = c.q.shape[0], c.table.shape
    table = torch.zeros((B + 2, columns + 8), dtype=torch.int32, device=DEV)
    table[1:B + 1, 4:4 + columns] = c.table
    O, _, tol, _ = c.reference()

    def attend_(q_start, kv_len, max_new):
        out, lse = torch.full((T + 4,) + c.q.shape[1:], 7.0, dtype=c.q.dtype, device=DEV), torch.full((T + 4, c.Hq), 7.0, device=DEV)
        lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, table[1:B + 1, 4:4 + columns], kv_len, q_start, out=out[2:T + 2], lse=lse[2:T + 2], max_new=max_new)
        torch.cuda.synchronize()
        for edge in (out[:2], out[T + 2:], lse[:2], lse[T + 2:]):
            assert (edge == 7.0).all()
        return out[2:T + 2].cpu().double()

    for max_new in (40, T):
        wrong = c.kv_len.clone()
        wrong[1], wrong[3] = -5, 2 ** 31 - 1
        got = attend_(c.q_start, wrong, max_new)
        for b in (0, 2, 4):
            at = slice(c.starts[b], c.starts[b + 1])
            assert ((got[at] - O[at]).abs() <= tol[at]).all(), b
        for starts in ([0, 40, 2, 4, 9, 49], [5, 3, 1, 0, 0, 0], [-9, -2, 20, 90, 3, 1], [100, 200, 300, 400, 500, 600], [0, 2 ** 31 - 1, -2 ** 31, 7, 8, 9], [2] * 6):
            attend_(torch.tensor(starts, dtype=torch.int32, device=DEV), c.kv_len, max_new)
        assert ((attend_(c.q_start, c.kv_len, max_new) - O).abs() <= tol).all()   # the workspace serves the next call


BETWEEN = [(8, 3000), (5, 700), (1, 100), (6, 6), (7, 33), (4, 200), (0, 50), (8, 3), (3, 4000)]   # of 8 heads a KV head: up to 64 rows


@pytest.mark.parametrize("Hq,Hkv,D,layout,page", [(16, 2, 128, "head", 16), (8, 1, 128, "token", 64), (64, 8, 128, "head", 32), (16, 2, 64, "token", 16), (7, 1, 128, "head", 64)])
@pytest.mark.parametrize("holes", [False, True])
def test_up_to_64_rows_of_a_branch(lotts, Hq, Hkv, D, layout, page, holes):
    """Items of up to 32 and of up to 64 rows in a call, in one piece and cut."""
    new, length = zip(*BETWEEN)
    gone = [(0, 0, -1), (1, 2, 5), (8, 100 * 16 // page, -1), (3, 0, -7)] if holes else ()
    c = MxCache(new, length, Hq, Hkv, D, page, "bf16", layout, holes=gone, seed=Hq + D)
    check(c, *attend(lotts, c, max_new=8))
    first = attend(lotts, c, max_new=8)
    for a, b in zip(first, attend(lotts, c, max_new=8)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Hq,Hkv,D,page,layout", [(16, 2, 128, 16, "head"), (40, 5, 128, 32, "token"), (16, 2, 64, 16, "token")])
def test_nan_in_v_of_up_to_64_rows(lotts, Hq, Hkv, D, page, layout):
    """A block of NaN in V at keys that some of the new tokens see and some do not."""
    new, length = zip(*BETWEEN)
    c = MxCache(new, length, Hq, Hkv, D, page, "bf16", layout, seed=D)
    scales, off = c.Vs.view(torch.uint8), torch.zeros(c.q.shape, dtype=torch.bool)
    for b, (n, L) in enumerate(BETWEEN):
        first = L - n
        for i, key in enumerate(range(max(first, 0), L, 2)):
            h, block = i % Hkv, i % (D // 32)
            scales[int(c.table[b, key // page]), h, key % page, block] = 255
            c.v[b][key, h, block * 32:block * 32 + 32] = 0.0
            off[c.starts[b] + key - first:c.starts[b] + n, h * (Hq // Hkv):(h + 1) * (Hq // Hkv), block * 32:block * 32 + 32] = True
    O, _, tol, _ = c.reference()
    got = lotts.verify_attention_paged_mxfp8(c.Q, *c.cache, c.table, c.kv_len, c.q_start, max_new=8).cpu().double()
    assert torch.isnan(got[off]).all() and ((got - O).abs() <= tol)[~off].all()


@pytest.mark.parametrize("Hq,Hkv,page,most", [(32, 8, 32, 2), (8, 2, 16, 4), (12, 6, 64, 3), (16, 16, 16, 1), (32, 8, 16, 300)])
def test_heads_of_64_next_to_each_other(lotts, Hq, Hkv, page, most):
    """Tokens in front of heads: two heads' codes of a key lie in one line of memory, and their workers alternate.  Branches of all lengths, a few and many."""
    for B in (1, 9, 70):
        new = [1 + i % min(most, 4) for i in range(B)]
        if most > 4:
            new[B // 2] = most
        length = [n + (i * 911) % 1500 for i, n in enumerate(new)]
        c = MxCache(new, length, Hq, Hkv, 64, page, "bf16", "token", seed=B + Hq)
        check(c, *attend(lotts, c, max_new=max(new)))
