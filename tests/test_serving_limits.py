"""Sizes at which 8-bit serving's counts would leave their types: refused, or worked out right, on the host (no GPU needed)."""
import ctypes

import pytest

from test_serving_args import B, FAKE, _cache, _job  # noqa: F401


def _run(B, **k):
    return B.lib().cmpq_kv_attention(ctypes.byref(_job(B, **k)), None, 0, None)     # -5 (no workspace): not refused before


def _size(B, **k):
    return B.lib().cmpq_kv_attention_workspace(ctypes.byref(_job(B, **k)))


def test_columns_of_a_head_that_32_bits_do_not_count(B):
    one = _cache(B, kv_heads=1, head_dim=1)
    for n, heads in ((1 << 25, 128), (1 << 24, 128), (1 << 30, 2), ((1 << 31) - 1, 1)):
        assert _run(B, cache=one, n_seq=1, n_rows=n, max_rows=n, q_heads=heads) == -2, (n, heads)
        assert _size(B, cache=one, n_seq=1, n_rows=n, max_rows=n, q_heads=heads) == 0
        assert _run(B, cache=one, n_seq=1, n_rows=n, max_rows=3, q_heads=heads) == -5          # of no sequence so many
    assert _run(B, cache=one, n_seq=1, n_rows=(1 << 30) - 513, max_rows=1 << 30, q_heads=2) == -5


@pytest.mark.parametrize("max_length", [64, 5000, 1 << 20])
@pytest.mark.parametrize("max_rows", [1, 40, 3000])
def test_windows_that_no_length_reaches_are_none(B, max_length, max_rows):
    sizes = dict(max_length=max_length, max_rows=max_rows, n_rows=2 * max_rows, ld_table=1 << 15)
    want = _size(B, **sizes)
    for window in (1 << 31, 1 << 62, (1 << 63) - 40, (1 << 63) - 1):
        assert _size(B, window=window, **sizes) == want


def test_sizes_that_are_refused_have_no_workspace(B):
    for bad in (dict(max_length=1 << 31), dict(max_rows=1 << 31), dict(n_rows=1 << 31), dict(n_seq=1 << 31), dict(q_heads=5), dict(q_heads=1 << 17),
                dict(window=-1), dict(ld_table=-1), dict(cache=_cache(B, page=40)), dict(cache=_cache(B, kv_heads=0)), dict(n_seq=1 << 24)):
        assert _size(B, **bad) == 0, bad
    assert _run(B, n_seq=1 << 24) == -2
