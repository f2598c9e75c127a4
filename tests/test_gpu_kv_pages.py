"""The pages' upkeep and the append into pages against plain Python: the same table, references, lengths, copies and pairs, whole numbers all."""
import math
import random

import pytest
import torch

import paged_util as P
from paged_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


def gpu(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class State:
    """Table, references and lengths on the GPU and as lists; branches may share the pages of a common beginning."""

    def __init__(self, B, columns, pages, page, seed, share=True, longest=None):
        rng = random.Random(seed)
        self.page, self.refs = page, [0] * pages
        self.table, self.kv_len = [], []
        free = list(range(pages))
        rng.shuffle(free)
        for b in range(B):
            L = rng.randint(0, min(longest or columns * page, columns * page))
            row, need = [], -(-L // page)
            if share and self.table and rng.random() < 0.5:
                other = rng.randrange(b)
                row = self.table[other][:rng.randint(0, min(need, sum(e >= 0 for e in self.table[other])))]
            while len(row) < need and free:
                row.append(free.pop())
            L = min(L, len(row) * page)
            for e in row:
                self.refs[e] += 1
            self.table.append(row + [-1] * (columns - len(row)))
            self.kv_len.append(L)
        wide = torch.full((B, columns + 3), -5, dtype=torch.int32, device=DEV)   # rows apart
        self.wide, self.g_table = wide, wide[:, :columns]
        self.g_table.copy_(gpu(self.table))
        self.g_refs, self.g_len = gpu(self.refs), gpu(self.kv_len)

    def same(self):
        torch.cuda.synchronize()
        assert self.g_len.tolist() == self.kv_len
        assert self.g_table.tolist() == self.table
        assert self.g_refs.tolist() == self.refs
        assert (self.wide[:, self.g_table.shape[1]:] == -5).all()

    def reserve(self, lotts, new):
        copies, missing = lotts.kv_pages_reserve(self.g_table, self.g_refs, self.g_len, gpu(new), self.page)
        want, lacking = P.reserve(self.table, self.refs, self.kv_len, new, self.page)
        self.same()
        assert missing.tolist() == [lacking] and copies.tolist() == want
        return copies, lacking


SIZES = [(1, 1, 1, 16), (1, 300, 500, 16), (5, 9, 40, 64), (33, 20, 500, 16), (64, 130, 9000, 32), (200, 7, 1500, 1024), (1100, 3, 4000, 16), (4096, 2, 9000, 16),
         (3, 40, 70000, 128)]


@pytest.mark.parametrize("B,columns,pages,page", SIZES)
def test_reserve(lotts, B, columns, pages, page):
    print("reserve", B, columns, pages, page, flush=True)
    s = State(B, columns, pages, page, B + pages, longest=columns * page * 2 // 3)
    rng = random.Random(1)
    reached = set()
    for most in (1, 5, page, 3 * page, 3 * page):
        new = [rng.choice([0, rng.randint(0, most)]) for _ in range(B)]
        new = [min(n, columns * page - L) if rng.random() < 0.999 else n for n, L in zip(new, s.kv_len)]
        reached.add(s.reserve(lotts, new)[1] > 0)
    assert False in reached


def test_reserve_without_room_changes_nothing(lotts):
    s = State(4, 6, 12, 16, 3, longest=60)
    lacking = s.reserve(lotts, [90 - L for L in s.kv_len])[1]
    assert lacking > 0
    assert s.reserve(lotts, [0, 97 - s.kv_len[1], 0, 1])[1] == -1
    assert s.reserve(lotts, [0, 0, 0, 0])[1] == 0
    assert s.reserve(lotts, [-3, 0, 0, 2])[1] == 0


def test_reserve_replaces_pages_that_are_shared_and_hold_nothing_to_keep(lotts):
    """A branch rolled back in front of a shared page gets one of its own there, without a copy."""
    s = State(1, 4, 20, 16, 0, longest=0)
    s.table, s.kv_len, s.refs = [[3, 5, -1, -1], [3, 5, -1, -1], [3, 5, 7, -1]], [10, 20, 40], [0] * 20
    for row in s.table:
        for e in row:
            if e >= 0:
                s.refs[e] += 1
    s.wide = torch.full((3, 7), -5, dtype=torch.int32, device=DEV)
    s.g_table = s.wide[:, :4]
    s.g_table.copy_(gpu(s.table))
    s.g_refs, s.g_len = gpu(s.refs), gpu(s.kv_len)
    assert s.reserve(lotts, [10, 1, 30])[1] == -1   # 70 tokens in 4 columns
    copies, lacking = s.reserve(lotts, [10, 1, 24])
    assert lacking == 0 and copies.tolist() == [[3, 0], [5, 2], [-1, -1]] and s.table[2] == [3, 5, 7, s.table[2][3]]
    assert s.refs[5] == 1 and s.table[0][1] == 1


@pytest.mark.parametrize("B,columns,pages,page", SIZES)
def test_fork(lotts, B, columns, pages, page):
    print("fork", B, columns, pages, page, flush=True)
    s = State(B, columns, pages, page, B)
    rng = random.Random(2)
    for parent in ([rng.randint(-1, B) for _ in range(B)], list(range(B))[::-1], list(range(B)), [0] * B, [-1 - b for b in range(B)]):
        lotts.kv_pages_fork(s.g_table, s.g_refs, s.g_len, gpu(parent))
        P.fork(s.table, s.refs, s.kv_len, parent)
        s.same()
    assert not any(s.refs) and not any(s.kv_len)


@pytest.mark.parametrize("B,columns,pages,page", SIZES)
def test_free(lotts, B, columns, pages, page):
    print("free", B, columns, pages, page, flush=True)
    s = State(B, columns, pages, page, B + 1)
    rng = random.Random(3)
    keep = [rng.choice([L, L + 3, L - 1, rng.randint(-2, columns * page)]) for L in s.kv_len]
    lotts.kv_pages_free(s.g_table, s.g_refs, s.g_len, page, keep=gpu(keep))
    P.free(s.table, s.refs, s.kv_len, page, keep)
    s.same()
    s.kv_len = [L - rng.randint(0, L) for L in s.kv_len]   # rolled back by an acceptance
    s.g_len.copy_(gpu(s.kv_len))
    lotts.kv_pages_free(s.g_table, s.g_refs, s.g_len, page)
    P.free(s.table, s.refs, s.kv_len, page)
    s.same()
    lotts.kv_pages_free(s.g_table, s.g_refs, s.g_len, page, keep=gpu([0] * B))
    P.free(s.table, s.refs, s.kv_len, page, [0] * B)
    s.same()
    assert not any(s.refs)


@pytest.mark.parametrize("B,columns,pages,page", SIZES)
def test_compact(lotts, B, columns, pages, page):
    print("compact", B, columns, pages, page, flush=True)
    s = State(B, columns, pages, page, B + 2)
    rng = random.Random(4)
    planes, width = 3, 24
    pool = torch.randint(0, 1 << 30, (planes, pages, width), dtype=torch.int32, device=DEV)
    for _ in range(2):
        keep = [L if rng.random() < 0.6 else rng.randint(0, L) for L in s.kv_len]
        lotts.kv_pages_free(s.g_table, s.g_refs, s.g_len, page, keep=gpu(keep))
        P.free(s.table, s.refs, s.kv_len, page, keep)
        before = pool.clone()
        held = [[before[:, e].clone() for e in row if e >= 0] for row in s.table[:20]]
        moves, counts = lotts.kv_pages_compact(s.g_table, s.g_refs)
        lotts.kv_pages_copy(pool, moves, count=counts)
        pairs, live = P.compact(s.table, s.refs)
        s.same()
        assert counts.tolist() == [len(pairs), live] and moves[:len(pairs)].tolist() == pairs
        assert all(r > 0 for r in s.refs[:live]) and not any(s.refs[live:])
        for row, was in zip(s.table, held):
            for e, data in zip([e for e in row if e >= 0], was):
                assert torch.equal(pool[:, e], data)
        want = before
        for src, dst in pairs:
            want[:, dst] = before[:, src]
        assert torch.equal(pool, want)


@pytest.mark.parametrize("planes,pages,shape,dtype", [(1, 2, (8,), torch.bfloat16), (4, 9, (2, 16, 64), torch.bfloat16), (2, 40, (3, 32, 128), torch.float32),
                                                      (72, 30, (2, 16, 128), torch.bfloat16), (3, 5, (8, 1024, 128), torch.bfloat16), (2, 7, (1040,), torch.uint8)])
def test_copy(lotts, planes, pages, shape, dtype):
    print("copy", planes, pages, shape, flush=True)
    make = lambda: torch.randint(0, 120, (planes, pages + 2) + shape, device=DEV).to(dtype)
    big = make()
    pool, want = big[:, 1:pages + 1], big.clone()
    ids = torch.randperm(pages).tolist()
    pairs = [[ids[2 * j], ids[2 * j + 1]] for j in range(pages // 2)] + [[-1, 0], [0, pages], [pages + 5, -1], [ids[0], ids[0]], [2 ** 31 - 1, 0]]
    used = pairs[:pages // 2]
    lotts.kv_pages_copy(pool, gpu(pairs))
    for src, dst in used:
        want[:, 1 + dst] = want[:, 1 + src]
    assert torch.equal(big, want)
    fresh = make()
    big.copy_(fresh)
    for n in (0, 1, len(pairs) + 9, -4):
        lotts.kv_pages_copy(pool, gpu(pairs), count=gpu([n]))
        for src, dst in used[:max(0, n)]:
            fresh[:, 1 + dst] = fresh[:, 1 + src]
        assert torch.equal(big, fresh), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,D", [(1, 8), (2, 128), (8, 128), (16, 64), (5, 40), (40, 128)])
@pytest.mark.parametrize("B,page,layout", [(1, 16, "head"), (6, 64, "token"), (70, 16, "token"), (300, 32, "head")])
def test_append(lotts, B, page, layout, Hkv, D, dtype):
    print("append", B, page, layout, Hkv, D, dtype, flush=True)
    rng = random.Random(B + D)
    new = [rng.choice([0, 1, 3, rng.randint(0, 40)]) for _ in range(B)]
    new[0] = 37
    length = [n + rng.randint(0, 3 * page) for n in new]
    c = P.Cache(new, length, Hkv, Hkv, D, page, dtype, layout, seed=B)
    if B > 5:   # tokens in front of the branch, in no page, behind the table
        c.kv_len[1], c.table[2, 0], c.kv_len[3] = 1, -1, c.table.shape[1] * page + 2
        c.table[4, -1] = c.K.shape[0]
    T = sum(new)
    qkv = torch.randn(T + 1, 3 * Hkv, D, device=DEV).to(c.q.dtype)   # one row more than the branches have
    k, v = qkv[:, Hkv:2 * Hkv], qkv[:, 2 * Hkv:]
    want = [t.clone() for t in (c.K, c.V)]
    table, kv_len = c.table.tolist(), c.kv_len.tolist()
    for b in range(B):
        for i in range(new[b]):
            t = kv_len[b] - new[b] + i
            if t < 0 or t // page >= len(table[b]) or not 0 <= table[b][t // page] < c.K.shape[0]:
                continue
            want[0][table[b][t // page], :, t % page] = k[c.starts[b] + i]
            want[1][table[b][t // page], :, t % page] = v[c.starts[b] + i]
    lotts.kv_append_paged(k, v, c.K, c.V, c.table, c.kv_len, c.q_start)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    for got, ref in zip((c.K, c.V), want):
        assert torch.equal(got.contiguous().view(bits), ref.contiguous().view(bits))


def test_append_as_many_tokens_of_every_branch(lotts):
    B, n, Hkv, D, page = 7, 4, 2, 64, 16
    c = P.Cache([n] * B, [4 + 9 * b for b in range(B)], 8, Hkv, D, page, seed=5)
    d = P.Cache([n] * B, [4 + 9 * b for b in range(B)], 8, Hkv, D, page, seed=5)
    qkv = torch.randn(B, n, 8 + 2 * Hkv, D, device=DEV).to(torch.bfloat16)
    lotts.kv_append_paged(qkv[:, :, 8:8 + Hkv], qkv[:, :, 8 + Hkv:], c.K, c.V, c.table, c.kv_len)
    flat = qkv.view(B * n, -1, D)
    lotts.kv_append_paged(flat[:, 8:8 + Hkv], flat[:, 8 + Hkv:], d.K, d.V, d.table, d.kv_len, d.q_start)
    for a, b in ((c.K, d.K), (c.V, d.V)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    tail = c.kv_len.long() - 1
    at = c.table[torch.arange(B, device=DEV), tail // page].long()
    assert torch.equal(c.K[at, :, tail % page], qkv[:, -1, 8:8 + Hkv])


@pytest.mark.parametrize("captured", [False, True])
def test_a_generation(lotts, captured):
    """A prompt read in two chunks, forked into branches, steps of drafts with roll-backs, a branch that ends, a fork in mid generation, compaction:
    after every step the attention of the new tokens is that of the tokens that the branches hold, kept in plain lists."""
    B, Hq, Hkv, D, page, columns, pages, n = 6, 8, 2, 64, 16, 8, 40, 4
    rng, g = random.Random(7), torch.Generator().manual_seed(7)
    pool = torch.full((2, pages, Hkv, page, D), math.nan, dtype=torch.bfloat16, device=DEV)
    table = torch.full((B, columns), -1, dtype=torch.int32, device=DEV)
    refs, kv_len = torch.zeros(pages, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    tokens = [[] for _ in range(B)]   # (k, v) of every token of a branch
    ws = torch.zeros(32 << 20, dtype=torch.uint8, device=DEV)
    new_t, q_start = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    T = 2 * page + 5
    qkv = torch.zeros(T, Hq + 2 * Hkv, D, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device=DEV), torch.zeros(T, Hq, device=DEV)
    copies, missing = torch.zeros(B, 2, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)

    def enqueue():
        lotts.kv_pages_reserve(table, refs, kv_len, new_t, page, copies=copies, missing=missing, workspace=ws)
        lotts.kv_pages_copy(pool, copies)
        lotts.kv_append_paged(qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], pool[0], pool[1], table, kv_len, q_start)
        lotts.verify_attention_paged(qkv[:, :Hq], pool[0], pool[1], table, kv_len, q_start, out=out, lse=lse, workspace=attn_ws)

    attn_ws = torch.zeros(256 << 20, dtype=torch.uint8, device=DEV)
    graph = None
    if captured:
        enqueue()   # with no new tokens: nothing changes
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            enqueue()

    def step(new):
        host = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(torch.bfloat16)
        qkv.copy_(host)
        new_t.copy_(gpu(new))
        q_start.copy_(gpu([sum(new[:b]) for b in range(B + 1)]))
        graph.replay() if captured else enqueue()
        torch.cuda.synchronize()
        assert missing.item() == 0
        ref = P.Cache(new, [len(t) + m for t, m in zip(tokens, new)], Hq, Hkv, D, page, device="cpu")
        ref.q = host[:sum(new), :Hq]
        for b in range(B):
            for i in range(new[b]):
                row = host[ref.starts[b] + i].double()
                tokens[b].append((row[Hq:Hq + Hkv], row[Hq + Hkv:]))
            for j, mine in enumerate((ref.k, ref.v)):
                mine[b] = torch.stack([t[j] for t in tokens[b]]) if tokens[b] else torch.zeros(0, Hkv, D, dtype=torch.float64)
        P.check(ref, out[:sum(new)], lse[:sum(new)])
        held = table[table >= 0].long()
        assert torch.equal(torch.bincount(held, minlength=pages), refs.long())
        assert kv_len.tolist() == [len(t) for t in tokens]

    def fork(parent):
        lotts.kv_pages_fork(table, refs, kv_len, gpu(parent))
        old = [list(t) for t in tokens]
        for b, f in enumerate(parent):
            tokens[b] = list(old[f]) if f >= 0 else []

    step([2 * page + 5, 0, 0, 0, 0, 0])
    step([7, 0, 0, 0, 0, 0])
    fork([0] * B)
    for turn in range(6):
        step([n] * B)
        accepted = [rng.randint(1, n) for _ in range(B)]
        for b in range(B):
            tokens[b] = tokens[b][:len(tokens[b]) - n + accepted[b]]
        kv_len.sub_(gpu([n - a for a in accepted]))
        if turn % 2:
            lotts.kv_pages_free(table, refs, kv_len, page)
        if turn == 2:
            fork([0, 0, -1, 3, 5, 4])
        if turn == 4:
            moves, counts = lotts.kv_pages_compact(table, refs)
            lotts.kv_pages_copy(pool, moves, count=counts)
            assert table.max().item() < counts[1].item()
    lotts.kv_pages_free(table, refs, kv_len, page, keep=torch.zeros(B, dtype=torch.int32, device=DEV))
    assert not refs.any() and not kv_len.any() and (table == -1).all()


def test_an_acceptance_rolls_the_lengths_back(lotts):
    """A step as a serving loop makes it: pages for the drafts, the acceptance takes the rejected ones off kv_len, their pages are given back."""
    B, k, V, page = 5, 3, 97, 16
    s = State(B, 9, 60, page, 11, longest=100)
    s.reserve(lotts, [k + 1] * B)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    zt = torch.randn(B, k + 1, V, generator=g, device=DEV)
    zd = zt[:, :k] + torch.randn(B, k, V, generator=g, device=DEV)
    draft = torch.randint(0, V, (B, k), generator=g, device=DEV, dtype=torch.int32)
    n, _ = lotts.spec_accept_logits(zt, zd, draft, torch.rand(B, k + 1, generator=g, device=DEV), priv_len=s.g_len)
    s.kv_len = [L - k + a for L, a in zip(s.kv_len, n.tolist())]
    lotts.kv_pages_free(s.g_table, s.g_refs, s.g_len, page)
    P.free(s.table, s.refs, s.kv_len, page)
    s.same()
    s.reserve(lotts, [k + 1] * B)


def test_on_another_stream(lotts):
    """The whole chain on a stream of its own, behind work that the current stream has nothing to do with."""
    stream = torch.cuda.Stream()
    s = State(4, 9, 80, 16, 12, longest=100)
    parent = [1, 1, 0, 3]
    stream.wait_stream(torch.cuda.current_stream())
    lotts.kv_pages_fork(s.g_table, s.g_refs, s.g_len, gpu(parent), stream=stream)
    torch.cuda.synchronize()   # (the argument's tensor was made on the current stream)
    new = gpu([5, 0, 20, 1])
    torch.cuda.synchronize()
    copies, missing = lotts.kv_pages_reserve(s.g_table, s.g_refs, s.g_len, new, 16, stream=stream)
    stream.synchronize()
    P.fork(s.table, s.refs, s.kv_len, parent)
    want, lacking = P.reserve(s.table, s.refs, s.kv_len, [5, 0, 20, 1], 16)
    s.same()
    assert copies.tolist() == want and missing.tolist() == [lacking]
