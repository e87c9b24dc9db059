"""Rows whose root lies halfway between two numbers of fp32, where the last bits of the sum of squares decide: the same for any
number of rows, as values and in 8 bits."""
import numpy as np
import pytest
import torch

import feed_forward_reference as Q
import serving_reference as R
from test_gpu_rms_norm import DEV, EPS, S  # noqa: F401

pytestmark = pytest.mark.gpu


def _halfway(rows, d, seed):
    """Rows of fp32 whose 1 / sqrt(mean + eps) is a midpoint within 2^-60 of itself: three elements make up what is missing."""
    g = np.random.default_rng(seed)
    X = g.standard_normal((rows, d)).astype(np.float32)
    X[:, [5, 77, d - 1]] = 0
    q = np.square(X.astype(np.longdouble)).sum(1)
    r = (1 / np.sqrt(q / d + np.longdouble(EPS))).astype(np.float32)
    low = np.nextafter(r, np.float32(0))
    low = np.nextafter(low, np.float32(0))
    mid = (low.astype(np.longdouble) + np.nextafter(low, np.float32(2)).astype(np.longdouble)) / 2
    want = (1 / np.square(mid) - np.longdouble(EPS)) * d
    for at in (5, 77, d - 1):
        x = np.nextafter(np.sqrt(want - q).astype(np.float32), np.float32(0))
        X[:, at] = x
        q = q + np.square(x.astype(np.longdouble))
    assert (np.abs(q - want) <= 2.0 ** -58 * want).all()
    return X


@pytest.mark.parametrize("d", [4104, 5000, 6144, 6200, 8000, 8192])
def test_rows_do_not_depend_on_how_many_there_are(S, d):  # noqa: F811
    X = torch.from_numpy(_halfway(64, d, d)).to(DEV)
    many = X.repeat(9, 1)                                                     # from 512 rows on the 8-bit form has other kernels
    Y = S.rms_norm(X, None, EPS)
    assert torch.equal(S.rms_norm(many, None, EPS), Y.repeat(9, 1))
    codes, scale = R.rows_in_8_bits(Y.cpu().numpy())
    for rows, times in ((S.rms_norm(X, None, EPS, coded=True), 1), (S.rms_norm(many, None, EPS, coded=True), 9)):
        got = Q.coded(rows)
        assert np.array_equal(got[1], np.tile(scale, times)) and np.array_equal(got[0], np.tile(codes, (times, 1)))
