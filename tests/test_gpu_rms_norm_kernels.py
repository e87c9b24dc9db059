"""Sizes and types that between them launch every kernel of the norm: 4 or 16 wavefronts a row, 1 to 4 steps, rows read again;
all tensors of one type or not; rows in 8 bits of many rows."""
import pytest
import torch

import test_gpu_rms_norm as T
from test_gpu_rms_norm import S  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("dtype", T.TYPES)
@pytest.mark.parametrize("m,d", [(5, 2000), (5, 4000), (5, 5000), (5, 7000), (5, 12000), (5, 30001), (3, 50000), (600, 4500), (520, 6144), (515, 6145),
                                 (700, 8191), (512, 4097), (511, 5001)])
def test_one_type(S, m, d, dtype):  # noqa: F811
    X, A, W = (T._randn(i, *s, dtype=dtype) for i, s in ((1, (m, d)), (2, (m, d)), (3, (d,))))
    T._check(S, X, W, A)
    T._check(S, X)


@pytest.mark.parametrize("m,d", [(600, 5000), (530, 8192), (3, 8000), (2, 20000)])
def test_two_types(S, m, d):  # noqa: F811
    X, A, W = T._randn(1, m, d, dtype=torch.bfloat16), T._randn(2, m, d), T._randn(3, d, dtype=torch.float16)
    T._check(S, X, W, A)
    T._check(S, X, W, A, torch.float32, torch.float16)


def test_rows_in_8_bits_do_not_depend_on_how_many_there_are(S):  # noqa: F811
    for d in (300, 3000, 5000, 8000):
        X = T._randn(1, 700, d, dtype=torch.bfloat16)
        whole = T.Q.coded(S.rms_norm(X, coded=True))
        for n in (1, 7, 300):
            part = T.Q.coded(S.rms_norm(X[:n], coded=True))
            assert (part[0] == whole[0][:n]).all() and (part[1] == whole[1][:n]).all()
