"""verify_attention_paged on device data outside its contract -- lengths that no table holds, first rows that do not ascend --: nothing outside the
outputs' rows changes, and where only lengths are wrong the other branches' rows are what they would be without."""
import pytest
import torch

from paged_util import DEV, Cache, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


def guarded(c):
    """The cache's table as rows of a wider buffer that names page 0 all around, O and lse between rows of their own."""
    B, columns = c.table.shape
    wide = torch.zeros((B + 2, columns + 8), dtype=torch.int32, device=DEV)
    wide[1:B + 1, 4:4 + columns] = c.table
    T = c.q.shape[0]
    out = torch.full((T + 4,) + c.q.shape[1:], 7.0, dtype=c.q.dtype, device=DEV)
    lse = torch.full((T + 4, c.Hq), 7.0, device=DEV)
    return wide[1:B + 1, 4:4 + columns], out, lse


def attend(lotts, c, q_start, kv_len, max_new):
    table, out, lse = guarded(c)
    T = c.q.shape[0]
    before = [t.clone().view(torch.uint8) for t in (c.K.contiguous(), c.V.contiguous(), c.Q)]
    lotts.verify_attention_paged(c.Q, c.K, c.V, table, kv_len, q_start, out=out[2:T + 2], lse=lse[2:T + 2], max_new=max_new)
    torch.cuda.synchronize()
    for edge in (out[:2], out[T + 2:], lse[:2], lse[T + 2:]):
        assert (edge == 7.0).all()
    for was, t in zip(before, (c.K.contiguous(), c.V.contiguous(), c.Q)):
        assert torch.equal(was, t.view(torch.uint8))
    return out[2:T + 2], lse[2:T + 2]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 40])
def test_lengths_that_no_table_holds(lotts, n, dtype):
    print("lengths", n, dtype, flush=True)
    c = Cache([n, 2, 1, n, 2], [200, 30, 90, 64, 150], 8, 2, 64, 16, dtype, seed=n)
    wrong = c.kv_len.clone()
    wrong[1], wrong[3] = -5, 2 ** 31 - 1
    out, lse = attend(lotts, c, c.q_start, wrong, n)
    O, _, tol, _ = c.reference()
    for b in (0, 2, 4):
        at = slice(c.starts[b], c.starts[b + 1])
        assert ((out[at].cpu().double() - O[at]).abs() <= tol[at]).all(), b
        assert torch.isfinite(lse[at]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("starts", [[0, 40, 2, 4], [0, 2, 40, 3], [5, 3, 1, 0], [-9, -2, 20, 90], [100, 200, 300, 400], [0, 2 ** 31 - 1, -2 ** 31, 7], [2, 2, 2, 2]], ids=str)
def test_first_rows_that_do_not_ascend(lotts, starts, dtype):
    print("starts", starts, dtype, flush=True)
    c = Cache([30, 4, 6], [64, 50, 64], 8, 2, 64, 16, dtype, more_columns=0, seed=1)   # the longest branches fill the table
    for max_new in (40, 6):
        attend(lotts, c, torch.tensor(starts, dtype=torch.int32, device=DEV), c.kv_len, max_new)
    check(c, *attend(lotts, c, c.q_start, c.kv_len, 30))   # the workspace serves the next call


def test_many_branches_whose_first_rows_do_not_ascend(lotts):
    """Beyond 64 branches the search has two steps."""
    c = Cache([1] * 130, [16] * 130, 4, 2, 64, 16, "f32", more_columns=0, seed=2)
    starts = torch.arange(131, dtype=torch.int32, device=DEV)
    for order in (starts.flip(0), torch.cat([starts[66:], starts[:66]]), starts * 3 % 131):
        attend(lotts, c, order.contiguous(), c.kv_len, 1)
    check(c, *attend(lotts, c, c.q_start, c.kv_len, 1))
