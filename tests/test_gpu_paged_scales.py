"""verify_attention_paged under scales whose products with the scores are beyond fp32: the largest score's key has all the weight, whatever its sign."""
import pytest
import torch

from paged_util import DEV, Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lotts():
    import paper_2505_19634_amd as m
    return m


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("new", [(1, 4), (20, 2), (300, 1)], ids=str)
def test_one_key_has_all_the_weight(lotts, new, sign, dtype):
    """Scores are whole numbers from 1 to 4096 or from -4096 to -1, all different along a row: a bf16 each in two terms, summed without rounding."""
    c = Cache(new, [n + 700 for n in new], 8, 2, 128, 16, dtype, seed=9)
    c.Q.zero_()
    c.Q[..., :3] = 1.0
    where = torch.arange(c.K.shape[0] * 16, device=DEV).reshape(c.K.shape[0], 16) * 37 % 4096
    K = torch.zeros_like(c.K)
    K[..., 0] = (where // 64 * 64).to(K.dtype)[:, None]
    K[..., 1] = (where % 64).to(K.dtype)[:, None]
    K[..., 2] = 1.0 if sign > 0 else -4096.0
    score = (where + (1 if sign > 0 else -4096)).tolist()
    table, length, V = c.table.tolist(), c.kv_len.tolist(), c.V.cpu()
    for scale in (1e3, 3e34, 1e36, 3e38):
        out, lse = lotts.verify_attention_paged(c.Q, K, c.V, c.table, c.kv_len, c.q_start, scale=scale, max_new=max(new), return_lse=True)
        out, lse = out.cpu(), lse.cpu()
        t = 0
        for b, n in enumerate(new):
            for i in range(n):
                best = max(range(length[b] - n + i + 1), key=lambda k: score[table[b][k // 16]][k % 16])
                assert torch.equal(out[t], V[table[b][best // 16], :, best % 16].repeat_interleave(4, dim=0)), (scale, b, i)
                top = score[table[b][best // 16]][best % 16]
                # rounded: the scale, its product with log2(e), that with the score, the sum with log2 of 1, the product with ln 2 and that constant: six half
                # steps of 2^-24; beyond fp32 it is an infinity of its sign
                if abs(top) * scale < 1e38:
                    assert (lse[t] - top * scale).abs().max() <= 8 * 2.0 ** -24 * abs(top) * scale
                else:
                    assert ((lse[t] > 1e37) if sign > 0 else (lse[t] < -1e37)).all()
                t += 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_as_small_as_the_scale_is_large(lotts, dtype):
    """Scores of some 2^-110 under a scale of 2^110 are scores of about 1."""
    c = Cache([3, 2], [300, 90], 8, 2, 128, 16, dtype, seed=4)
    plain = lotts.verify_attention_paged(c.Q, c.K, c.V, c.table, c.kv_len, c.q_start, scale=0.125, max_new=3)
    small = lotts.verify_attention_paged(c.Q * 2.0 ** -110, c.K, c.V, c.table, c.kv_len, c.q_start, scale=2.0 ** 107, max_new=3)
    assert torch.equal(plain, small)   # (powers of two: not a bit differs)
