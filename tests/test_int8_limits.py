"""Sizes of 8-bit products whose double leaves 64 bits: refused on the host like all beyond the limits (no GPU needed)."""
import ctypes

import pytest

from test_feed_forward_args import B, FAKE  # noqa: F401

HUGE = [1 << 23, 1 << 24, 1 << 61, 1 << 62, (1 << 62) + 16, (1 << 62) + (1 << 20), (1 << 63) - 1]


@pytest.mark.parametrize("d_out", HUGE)
def test_gated_outputs_beyond_the_limit(B, d_out):  # noqa: F811
    L = B.lib()
    assert B.int8_gated_rows(d_out) == 0
    assert L.cmpq_int8_prepare_gated(FAKE, FAKE, 0, d_out, 8, 8, 8, FAKE, FAKE, None, None) == -2
    for x in (dict(X=FAKE, ldx=8), dict(x_codes=FAKE, x_scale=FAKE)):
        job = B.Int8Job(m=4, d_in=8, codes=FAKE, scale=FAKE, d_out=d_out, gated=1, Y=FAKE, ldy=d_out, **x)
        assert L.cmpq_int8_product_job(ctypes.byref(job), FAKE, 1 << 30, None) == -2
