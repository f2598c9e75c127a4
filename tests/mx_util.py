"""What the tests of the microscaled numbers share: the format from its definition -- every element is looked up among all that there are --, and a paged
cache of such numbers."""
import math

import numpy as np
import torch

from paged_util import DEV, Cache

BLOCK = 32


def e4m3(code):
    e, m = code >> 3, code & 7
    return math.ldexp(1 + m / 8, e - 7) if e else math.ldexp(m / 8, -6)


KINDS = {  # elements of the codes 0, 1, ... without a sign; the bit of the sign; smallest and largest exponent of a scale
    "mxfp8": (np.array([e4m3(c) for c in range(127)]), 0x80, -117, 119),
    "mxfp4": (np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6]), 8, -125, 125),
}


def quantise(x, kind):
    """x [..., K] -> codes [..., K] (one in a byte, whatever the kind) and scale bytes [..., K / 32], numpy uint8."""
    elements, sign, lo, hi = KINDS[kind]
    x = np.asarray(x.double().numpy() if isinstance(x, torch.Tensor) else x, dtype=np.float64)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // BLOCK, BLOCK))
    bad = ~np.isfinite(b).all(-1)
    size = np.where(bad[..., None], 0.0, np.abs(b))
    most = size.max(-1)
    e = np.frexp(most)[1] - np.frexp(elements[-1])[1]     # at most one too small
    e = np.where(most > elements[-1] * np.ldexp(1.0, e), e + 1, e)
    e = np.clip(np.where(most == 0, lo, e), lo, hi)
    y = np.minimum(np.ldexp(size, -e[..., None]), elements[-1])
    above = np.searchsorted(elements, y)                  # the first element that is not smaller
    below = np.maximum(above - 1, 0)
    up, down = elements[above] - y, y - elements[below]
    code = np.where((up < down) | ((up == down) & (above % 2 == 0)) | (above == below), above, below)
    code = code + sign * np.signbit(b)
    code = np.where(bad[..., None], 0x7f if kind == "mxfp8" else 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales, kind):
    """What codes (one in a byte) and scale bytes stand for, float64."""
    elements, sign, _, _ = KINDS[kind]
    table = np.full(256, math.nan)
    table[:len(elements)] = elements
    table[sign:sign + len(elements)] = -elements
    two = np.where(scales == 255, math.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return table[codes] * np.repeat(two, BLOCK, -1)


def pack(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))


class MxCache(Cache):
    """A cache whose K and V are held in MXFP8: Kc, Vc codes, Ks, Vs scales, in the given order in memory; what no branch holds is NaN.  k and v are the
    values that the codes stand for."""

    def __init__(self, new, length, Hq, Hkv, D, page, dtype="bf16", layout="head", device=DEV, types=(torch.float8_e4m3fn, torch.float8_e8m0fnu), **other):
        super().__init__(new, length, Hq, Hkv, D, page, dtype, layout, device=device, **other)
        self.layout, self.types, self.device = layout, types, device
        self.Kc, self.Ks = self.held(self.K)
        self.Vc, self.Vs = self.held(self.V)
        self.k, self.v = ([torch.from_numpy(values(*quantise(t, "mxfp8"), "mxfp8")) for t in ts] for ts in (self.k, self.v))
        del self.K, self.V

    def held(self, pages):
        codes, scales = quantise(pages.cpu().float(), "mxfp8")

        def lay(a, dtype):
            t = torch.from_numpy(a)
            if self.layout == "token":
                t = t.transpose(1, 2).contiguous().to(self.device).transpose(1, 2)
            return t.to(self.device).view(dtype)
        return lay(codes, self.types[0]), lay(scales, self.types[1])

    @property
    def cache(self):
        return self.Kc, self.Vc, self.Ks, self.Vs
