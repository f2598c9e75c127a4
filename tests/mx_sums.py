"""Products of MXFP4 weights whose sums are exact in fp32 whatever their order: tokens are whole numbers up to 4, weights whole numbers up to 24, so that K of them
sum up to less than 2^24.  The result is then the exact one rounded to bf16 once, and a share of K that is lost or counted twice shows in it however long K is."""
import torch

LARGEST = 4 * 24
ELEMENTS = [0, 1, 2, 3, 4, 6]          # the whole numbers among e2m1, by their codes
CODES = [0, 2, 4, 5, 6, 7]


def whole_product(M, N, K, seed=0, device="cpu"):
    """X [M][K] bf16, codes [N][K / 2] and scales [N][K / 32] bytes, and the weights that these stand for, fp64."""
    assert K * LARGEST < 1 << 24 and K % 32 == 0
    g = torch.Generator(device=device).manual_seed(seed + M + N + K)
    pick = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device=device)
    X = pick(-4, 5, M, K).bfloat16()
    code = torch.tensor(CODES, device=device)[pick(0, 6, N, K)] + 8 * pick(0, 2, N, K)
    scales = pick(127, 130, N, K // 32)
    table = torch.tensor([0.0] * 8, dtype=torch.float64, device=device)
    table[CODES] = torch.tensor(ELEMENTS, dtype=torch.float64, device=device)
    w = torch.cat([table, -table])[code] * torch.exp2((scales - 127).double()).repeat_interleave(32, 1)
    return X, (code[:, 0::2] | code[:, 1::2] << 4).to(torch.uint8), scales.to(torch.uint8), w


def rounded(Y):
    """Whole numbers below 2^24, exact in fp32, to bf16."""
    return Y.float().bfloat16()
