"""verify_attention_paged against its definition in 64 bits: chunks, drafts and single tokens beside each other, branches without new tokens or
without any, pages of every size in either order, missing pages, rows that see nothing, and NaN in every place that no branch holds."""
import pytest
import torch

from paged_util import DEV, Cache, check

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
    lotts.verify_attention_paged(Q, c.K, c.V, c.table, c.kv_len, c.q_start, scale=scale, out=out, lse=lse, max_new=max_new, workspace=workspace)
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
HEADS = [(16, 2, 128), (8, 8, 64), (5, 1, 128), (28, 4, 64), (3, 3, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,page", [("head", 16), ("token", 64)])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("mix", sorted(MIXES))
def test_against_64_bits(lotts, mix, Hq, Hkv, D, layout, page, dtype):
    print("paged attention", mix, Hq, Hkv, D, layout, page, dtype, flush=True)
    new, length = zip(*MIXES[mix])
    c = Cache(new, length, Hq, Hkv, D, page, dtype, layout, seed=len(mix) + Hq)
    check(c, *attend(lotts, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
@pytest.mark.parametrize("n,L", [(1, 2049), (3, 5000), (17, 1500), (70, 1111)])
def test_lengths(lotts, n, L, page, dtype):
    print("paged attention", n, L, page, dtype, flush=True)
    c = Cache([n, 1], [L, L // 3], 4, 2, 64 if page == 32 else 128, page, dtype, seed=n)
    check(c, *attend(lotts, c, max_new=n))


@pytest.mark.parametrize("B", [63, 64, 65, 128, 130, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_branches(lotts, B, dtype):
    print("paged attention", B, dtype, flush=True)
    new = [(b * 7) % 4 for b in range(B)]
    length = [n + (b * 37) % 90 for b, n in enumerate(new)]
    c = Cache(new, length, 4, 2, 64, 16, dtype, seed=B)
    check(c, *attend(lotts, c, max_new=3))


@pytest.mark.parametrize("tiny", [3, 100, 400])
@pytest.mark.parametrize("chunk,L", [(90, 90), (150, 1000), (700, 3100)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_chunk_beside_tiny_branches(lotts, tiny, chunk, L, D):
    """The work's equal pieces may be as small as a tile of the chunk is long: every one of them has a part of it."""
    print("paged attention", tiny, chunk, L, D, flush=True)
    new = [1 + b % 2 for b in range(tiny // 2)] + [chunk] + [1] * (tiny - tiny // 2)
    length = [n + b % 3 for b, n in enumerate(new)]
    length[tiny // 2] = L
    c = Cache(new, length, 4, 2 if tiny < 100 else 1, D, 16, seed=tiny + chunk)
    check(c, *attend(lotts, c, max_new=chunk))


@pytest.mark.parametrize("n,L,Hq,Hkv", [(300, 300, 16, 2), (1030, 1500, 8, 8), (513, 4000, 5, 1), (2039, 2039, 16, 2), (260, 9000, 2, 1)])
def test_prompts(lotts, n, L, Hq, Hkv):
    """Items that are cut one by one, a few parts each."""
    print("paged attention", n, L, Hq, Hkv, flush=True)
    c = Cache([n], [L], Hq, Hkv, 128 if Hq != 5 else 64, 64, seed=n)
    check(c, *attend(lotts, c, max_new=n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32, 64])
def test_missing_pages(lotts, page, dtype):
    print("paged attention, missing pages", page, dtype, flush=True)
    holes = [(0, 0, -1), (0, 3, 0), (1, 1, -7), (2, 0, -1), (2, 1, 2 ** 30), (3, 5, -1), (3, 6, -1)]
    c = Cache([2, 80, 3, 1], [4 * page + 5, 2 * page + 9, 2 * page, 9 * page], 8, 2, 128, page, dtype, holes=holes, seed=page)
    check(c, *attend(lotts, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_as_many_tokens_of_every_branch(lotts, dtype):
    """Without q_start, Q [B][n][Hq][D] a view of a projection's output, out one of a larger buffer."""
    B, n, Hq, Hkv, D = 6, 3, 10, 2, 64
    c = Cache([n] * B, [40, 3, 129, 77, 64, 15], Hq, Hkv, D, 32, dtype, seed=3)
    qkv = torch.full((B * n, Hq + 2 * Hkv, D), float("nan"), dtype=c.q.dtype, device=DEV)
    qkv[:, :Hq] = c.Q
    big = torch.full((B, n, Hq + 1, D), 7.0, dtype=c.q.dtype, device=DEV)
    out, lse = lotts.verify_attention_paged(qkv.view(B, n, Hq + 2 * Hkv, D)[:, :, :Hq], c.K, c.V, c.table, c.kv_len, out=big[:, :, :Hq], return_lse=True)
    assert out.shape == (B, n, Hq, D) and lse.shape == (B * n, Hq)
    check(c, out, lse)
    assert (big[:, :, Hq] == 7.0).all()
    flat = lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len)
    assert torch.equal(flat.view(B, n, Hq, D), out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.03, 0.5])
def test_scale_and_wide_scores(lotts, scale, dtype):
    """Scores of some hundreds: nearly all weight on one key."""
    c = Cache([3, 50], [300, 210], 4, 2, 128, 16, dtype, seed=8, std=3.0)
    check(c, *attend(lotts, c, scale=scale), scale=scale)


def test_against_the_dense_cache(lotts):
    """The same keys in verify_attention's private caches: the same attention."""
    B, n, Hq, Hkv, D, L = 5, 4, 16, 2, 128, 700
    length = [700, 4, 333, 64, 511]
    c = Cache([n] * B, length, Hq, Hkv, D, 16, seed=2)
    K, V = (torch.zeros(B, Hkv, L, D, dtype=torch.bfloat16) for _ in range(2))
    for b in range(B):
        K[b, :, :length[b]], V[b, :, :length[b]] = c.k[b].transpose(0, 1), c.v[b].transpose(0, 1)
    dense, lse = lotts.verify_attention(c.Q.view(B, n, Hq, D), None, None, K.to(DEV), V.to(DEV), c.kv_len, return_lse=True)
    check(c, dense, lse)
    check(c, *attend(lotts, c))


def test_a_cache_beyond_4_gib(lotts):
    """Pages behind 2^32 bytes of the pool."""
    page, Hkv, D = 64, 8, 128
    pages = (5 << 30) // (Hkv * page * D * 2)
    K = torch.zeros((pages, Hkv, page, D), dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    c = Cache([3, 40], [300, 120], 16, Hkv, D, page, seed=4)
    far = torch.arange(c.K.shape[0], device=DEV, dtype=torch.int32) + (pages - c.K.shape[0])
    K[far.long()], V[far.long()] = c.K, c.V
    c.table = torch.where(c.table >= 0, c.table + (pages - c.K.shape[0]), c.table)
    c.K, c.V = K, V
    check(c, *attend(lotts, c))


def test_replays(lotts):
    """Captured once, replayed with other lengths, other pages and other numbers of new tokens."""
    first = Cache([2, 30, 1], [100, 64, 257], 16, 2, 128, 16, seed=0, spare_pages=40, more_columns=30)
    ws = torch.zeros(256 << 20, dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(first.Q)
    lse = torch.zeros(first.q.shape[:2], device=DEV)
    call = lambda: lotts.verify_attention_paged(first.Q, first.K, first.V, first.table, first.kv_len, first.q_start, out=out, lse=lse, max_new=32,
                                                workspace=ws)
    call()
    torch.cuda.synchronize()
    check(first, out, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed, (new, length) in enumerate([((2, 30, 1), (100, 64, 257)), ((1, 0, 32), (500, 0, 90)), ((31, 1, 1), (31, 333, 16)), ((2, 30, 1), (5, 450, 3))]):
        other = Cache(new, length, 16, 2, 128, 16, seed=seed + 50)
        for mine, its in ((first.K, other.K), (first.V, other.V)):
            mine[:its.shape[0]] = its
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
        lotts.verify_attention_paged(first.Q, first.K, first.V, first.table, first.kv_len, first.q_start, out=eager, max_new=32, workspace=ws)
        assert torch.equal(eager, out)


def test_streams_with_workspaces_of_their_own(lotts):
    """Calls that overlap in time, one a stream, and then all of them on one stream with one workspace: the same bits."""
    cases = [Cache(new, length, 16, 2, 128, 16, seed=i) for i, (new, length) in enumerate([((3, 1), (900, 4000)), ((300, 2), (700, 2500)), ((9, 9, 9), (100, 3000, 50))])]
    streams = [torch.cuda.Stream() for _ in cases]
    one = [lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, max_new=max(c.new), return_lse=True) for c in cases]
    torch.cuda.synchronize()
    outs = [torch.zeros_like(c.Q) for c in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, st, o in zip(cases, streams, outs):
            lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, max_new=max(c.new), out=o, stream=st)
    torch.cuda.synchronize()
    for c, (a, lse), b in zip(cases, one, outs):
        assert torch.equal(a, b)
        check(c, a, lse)


def test_a_workspace_that_an_unfinished_call_left(lotts):
    """Cells with an old tag and a count, anything in the partials: as good as zeros."""
    c = Cache([4, 300], [3000, 1500], 16, 2, 128, 16, seed=1)
    clean = attend(lotts, c, max_new=300)
    ws = torch.randint(0, 2 ** 31, (64 << 20,), dtype=torch.int32, device=DEV)
    ws[:4096] = torch.tensor([(1 << 16) + 3, 0], dtype=torch.int32, device=DEV).repeat(2048)   # 64-bit cells: tag 1, three arrivals
    dirty = attend(lotts, c, max_new=300, workspace=ws.view(torch.uint8))
    for a, b in zip(clean, dirty):
        assert torch.equal(a, b)


def test_max_new_is_a_bound_alone(lotts):
    """Known or not, the same attention; where the most new tokens are few the lighter kernel runs, whose pieces differ."""
    c = Cache([1, 4, 0, 2], [500, 90, 70, 1300], 8, 2, 64, 32, seed=6)
    for most in (None, 4, 5, 7):
        check(c, *attend(lotts, c, max_new=most))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(1, 4), (20, 2), (300, 1)], ids=str)
def test_a_scale_that_leaves_nothing_of_the_scores(lotts, new, dtype):
    """Scales whose reciprocal is beyond fp32 are scales: every key weighs the same."""
    c = Cache(new, [n + 700 for n in new], 8, 2, 128, 16, dtype, seed=8)
    for scale in (1e-38, 2e-39):
        check(c, *attend(lotts, c, scale=scale, max_new=max(new)), scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(1, 4), (20, 2), (300, 1)], ids=str)
def test_a_scale_that_leaves_one_key(lotts, new, dtype):
    """The larger the scale, the more the largest score's key has of the weight; from some point on it has all.  Scores are whole numbers, summed without
    rounding and all different along a row, so that the key is known and its value comes out as it is."""
    c = Cache(new, [n + 700 for n in new], 8, 2, 128, 16, dtype, seed=9)
    c.Q.zero_()
    c.Q[..., :2] = 1.0
    where = torch.arange(c.K.shape[0] * 16, device=DEV).reshape(c.K.shape[0], 16)
    K = torch.zeros_like(c.K)
    K[..., 0] = ((where * 37 % 4096) // 64 * 64).to(c.K.dtype)[:, None]   # multiples of 64 below 4096 and what is left: a bf16 each
    K[..., 1] = (where * 37 % 4096 % 64).to(c.K.dtype)[:, None]
    score = (where * 37 % 4096).tolist()
    table, length, V = c.table.tolist(), c.kv_len.tolist(), c.V.cpu()
    for scale in (1e3, 1e9, 1e30, 3e34):
        out = lotts.verify_attention_paged(c.Q, K, c.V, c.table, c.kv_len, c.q_start, scale=scale, max_new=max(new)).cpu()
        t = 0
        for b, n in enumerate(new):
            for i in range(n):
                best = max(range(length[b] - n + i + 1), key=lambda k: score[table[b][k // 16]][k % 16])
                want = V[table[b][best // 16], :, best % 16].repeat_interleave(4, dim=0)
                assert torch.equal(out[t], want), (scale, b, i)
                t += 1


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("most", [1, 5])
def test_more_items_than_twice_the_units(lotts, D, most):
    """More items than twice the units: two workgroups each; one branch is much longer than the others and is cut many times, some are empty."""
    new = [(i * 7) % (most + 1) for i in range(270)]
    length = [n + (i * 37) % 150 for i, n in enumerate(new)]
    new[100], length[100] = most, 9000
    c = Cache(new, length, 4, 2, D, 16, seed=D)
    check(c, *attend(lotts, c, max_new=most))


def test_one_workspace_for_every_kind_of_call(lotts):
    """Calls that lay their partials out differently take turns with one buffer; all of them cut branches."""
    many = Cache([1] * 260, [30] * 259 + [7000], 4, 2, 128, 16, seed=1)
    cases = [(many, 1), (Cache([300, 1], [2500, 900], 8, 2, 64, 16, seed=2), 300), (Cache([4, 2], [5000, 800], 8, 2, 128, 32, seed=3), 4),
             (Cache([12], [3000], 8, 2, 128, 16, seed=4), 12), (Cache([3, 1], [100, 60], 4, 2, 64, 16, "f32", seed=5), 3)]
    ws = torch.zeros(80 << 20, dtype=torch.uint8, device=DEV)
    first = [attend(lotts, c, max_new=n) for c, n in cases]
    for a, (c, _) in zip(first, cases):
        check(c, *a)
    for order in (range(5), (4, 3, 2, 1, 0), (1, 0, 3, 0, 2, 0, 4, 0)):
        for i in order:
            again = attend(lotts, cases[i][0], max_new=cases[i][1], workspace=ws)
            assert all(torch.equal(a, b) for a, b in zip(first[i], again)), i
