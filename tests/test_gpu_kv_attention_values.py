"""Attention over the paged cache where the values' sizes decide: near the top of a type's range, and of pages whose
scales lie many orders apart, judged row by row."""
import numpy as np
import pytest
import torch

import test_gpu_kv_attention as A

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


@pytest.mark.parametrize("dim", [32, 40, 64, 96, 160])
@pytest.mark.parametrize("rows", [1, 60])
def test_parts_of_large_values_are_added_once(S, dim, rows):
    """700 tokens of 2^111 with weights alike: the sum 2^7 * 700 * 2^111 that the parts are added to is below 2^128, twice as
    much is not.  Rounded on the way: weights of 1 not at all, the scale and the output's quotient in fp32 (2^-22 in all)
    and the output to bfloat16."""
    s = A.Bounded(S, [700], 1, dim, 32, dim)
    s.cache.v.fill_(255)
    s.cache.v_scale.fill_(2.0 ** 111 / 127)
    Q = torch.randn((rows, 2, dim), device=DEV).bfloat16()
    out = s.run(Q, [rows], softmax_scale=0.0)
    torch.cuda.synchronize()
    off = np.abs(out.double().cpu().numpy() / 2.0 ** 111 - 1)
    assert (off <= 2.0 ** -8 + 2.0 ** -22).all(), off.max()
