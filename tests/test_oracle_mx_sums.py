"""The products with exact sums notice every share of K: in the reference, a block that is left out or counted twice changes the result."""
import numpy as np
import pytest
import torch

from mx_sums import LARGEST, rounded, whole_product
from mx_util import unpack, values


def test_the_weights_are_what_codes_and_scales_stand_for():
    X, codes, scales, w = whole_product(2, 9, 1056)
    assert np.array_equal(values(unpack(codes.numpy()), scales.numpy(), "mxfp4"), w.numpy())
    assert (w.abs() <= LARGEST / 4).all() and (X.abs() <= 4).all() and (w == w.round()).all()


@pytest.mark.parametrize("M,N,K", [(1, 7, 28672), (3, 40, 16384), (70, 40, 27648)])
@pytest.mark.parametrize("share", [32, 256, 1024])
def test_every_share_shows(M, N, K, share):
    X, _, _, w = whole_product(M, N, K)
    x = X.double()
    Y = x @ w.t()
    assert torch.equal(Y, (x.float() @ w.float().t()).double())     # in whatever order fp32 sums them
    for k in range(0, K, share):
        part = x[:, k:k + share] @ w[:, k:k + share].t()
        assert not torch.equal(rounded(Y - part), rounded(Y)) and not torch.equal(rounded(Y + part), rounded(Y)), k
