"""The microscaled numbers that the GPU is checked against: pinned by torch's own 8-bit type, by hand, and by what the definition asks for."""
import numpy as np
import pytest
import torch

from mx_util import BLOCK, KINDS, pack, quantise, unpack, values


def test_elements_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    got = values(codes.numpy().reshape(8, 32), np.full((8, 1), 127, np.uint8), "mxfp8").reshape(256)
    assert np.array_equal(got, want, equal_nan=True) and np.array_equal(np.signbit(got[:255]), np.signbit(want[:255]))


def test_elements_round_as_torchs():
    """Blocks whose largest value is 448 have the scale 1."""
    g = np.random.default_rng(1)
    x = (g.standard_normal((400, 32)) * np.exp(g.uniform(-8, 5, (400, 1)))).clip(-448, 448)
    x[:, 3] = 448
    x = torch.from_numpy(x).float()
    codes, scales = quantise(x, "mxfp8")
    assert (scales == 127).all()
    assert np.array_equal(codes, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_four_bits_by_hand():
    x = np.zeros((1, 32))
    x[0, :12] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 0.26, -5.01, -0.0, -0.2]
    codes, scales = quantise(x, "mxfp4")
    assert scales.tolist() == [[127]]
    assert codes[0, :12].tolist() == [7, 0, 2, 2, 4, 4, 6, 6, 1, 15, 8, 8]


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_the_scale_is_the_smallest_and_every_element_the_nearest(kind):
    elements, sign, lo, hi = KINDS[kind]
    g = np.random.default_rng(2)
    x = g.standard_normal((2000, BLOCK)) * 2.0 ** g.integers(-140, 127, (2000, 1))
    codes, scales = quantise(x, kind)
    e = scales[:, 0].astype(int) - 127
    most = np.abs(x).max(-1)
    assert ((most <= elements[-1] * 2.0 ** e) | (e == hi)).all()
    assert ((most > elements[-1] * 2.0 ** (e - 1)) | (e == lo)).all()
    y = x / 2.0 ** e[:, None]
    off = np.abs(values(codes, np.full_like(scales, 127), kind) - y)
    assert (off <= np.abs(np.concatenate([elements, -elements])[None, None] - y[..., None]).min(-1) + 1e-12 * elements[-1])[e < hi].all()


def test_borders_and_what_is_no_number():
    for kind, (elements, sign, lo, hi) in KINDS.items():
        for p in range(-149, 128):   # the largest element times a power of two keeps its scale, anything more takes the next
            x = np.zeros((2, 32))
            x[0, 5] = np.ldexp(elements[-1], p - 3)
            x[1, 5] = np.nextafter(x[0, 5], np.inf)
            _, scales = quantise(x, kind)
            assert scales[0, 0] == np.clip(p - 3, lo, hi) + 127 and scales[1, 0] == np.clip(p - 2, lo, hi) + 127
        x = np.ones((3, 64))
        x[0, 3], x[1, 40] = np.inf, np.nan
        codes, scales = quantise(x, kind)
        v = values(codes, scales, kind)
        assert scales[0, 0] == 255 and scales[1, 1] == 255 and (scales == 255).sum() == 2
        assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:]).all() and (v[2] == 1).all() and (v[0, 32:] == 1).all()


def test_packing():
    c = np.arange(64, dtype=np.uint8).reshape(1, 64) % 16
    assert pack(c)[0, :3].tolist() == [0x10, 0x32, 0x54] and np.array_equal(unpack(pack(c)), c)
