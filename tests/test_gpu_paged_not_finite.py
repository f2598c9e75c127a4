"""verify_attention_paged with infinities and NaN in V: a row's output is not finite in the columns where a key that it sees is not, and the rows that do
not see the key are what they would be with anything else in its place."""
import math

import pytest
import torch

from paged_util import DEV, Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


MIXES = {  # (new tokens, all tokens) of the branches, and (branch, key counted from the branch's first new token, KV head, first column, value)
    "drafts": [(4, 100), (4, 4), (4, 65), (4, 513), (1, 40)],
    "two_row_tiles": [(16, 300), (9, 33), (12, 12)],
    "blind": [(5, 3), (40, 20), (3, 20), (70, 30)],
    "chunks": [(257, 700), (1, 1000), (60, 200), (300, 300)],
    "cut": [(6, 9000), (290, 4000)],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("Hq,Hkv,D,page,layout", [(16, 2, 128, 16, "head"), (4, 4, 64, 64, "token"), (6, 2, 128, 32, "token"), (8, 1, 64, 16, "head")])
@pytest.mark.parametrize("mix", sorted(MIXES))
def test_only_rows_that_see_the_key(lotts, mix, Hq, Hkv, D, page, layout, value, dtype):
    print("not finite", mix, Hq, Hkv, D, page, layout, value, dtype, flush=True)
    new, length = zip(*MIXES[mix])
    c = Cache(new, length, Hq, Hkv, D, page, dtype, layout, seed=len(mix) + D)
    g = torch.Generator().manual_seed(D + Hq)
    off = torch.zeros(c.q.shape, dtype=torch.bool)
    for b, (n, L) in enumerate(MIXES[mix]):
        first = L - n
        keys = {L - 1, max(0, first + n // 2), max(0, first), max(0, first + 1) if n > 1 else L - 1} - ({max(0, first)} if b % 2 else set())
        for key in sorted(keys):
            h = int(torch.randint(0, Hkv, (1,), generator=g))
            at = torch.randperm(D, generator=g)[:5]
            entry = int(c.table[b, key // page])
            c.V[entry, h, key % page, at.to(DEV)] = value
            c.v[b][key, h, at] = 0.0
            for i in range(max(0, key - first), n):
                rows = off[c.starts[b] + i, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)]
                rows[:, at] = True
    O, ref_lse, tol, tol_lse = c.reference()
    for max_new in {max(new), c.q.shape[0]}:
        out, lse = lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, max_new=max_new, return_lse=True)
        got, l = out.cpu().double(), lse.cpu().double()
        assert not torch.isfinite(got[off]).any()
        worst = ((got - O).abs() - tol)[~off].max().item()
        assert worst <= 0, worst   # (NaN is no number below 0)
        seen = ~torch.isinf(ref_lse)
        assert ((l - ref_lse).abs() <= tol_lse)[seen].all() and torch.isinf(l[~seen]).all()


def test_a_page_of_nothing_but_nan(lotts):
    """Every key of V is NaN: rows that see one are NaN, blind ones 0."""
    c = Cache([5, 40, 3], [3, 30, 200], 8, 2, 128, 16, seed=3)
    c.V.fill_(math.nan)
    for max_new in (40, 48):
        out = lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, max_new=max_new).cpu()
        blind = torch.zeros(48, dtype=torch.bool)
        blind[0:2] = blind[5:15] = True
        assert (out[blind] == 0).all() and torch.isnan(out[~blind]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_many_branches(lotts, D):
    """More items than twice the units, every second branch with an infinity in its last new token's V: the tokens in front of it are as without."""
    B, n = 300, 3
    c = Cache([n] * B, [n + (b * 37) % 90 for b in range(B)], 8, 2, D, 16, seed=D)
    clean = lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, max_new=n).view(B, n, 8, D)
    last = c.kv_len.long() - 1
    at = c.table[torch.arange(B, device=DEV), last // 16].long()
    c.V[at[::2], 1, last[::2] % 16, 5] = math.inf
    out = lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, max_new=n).view(B, n, 8, D)
    off = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
    off[::2, n - 1, 4:, 5] = True
    assert not torch.isfinite(out[off]).any() and torch.equal(out[~off], clean[~off])
