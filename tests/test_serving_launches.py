"""Caches and attention of more workgroups than a launch has lanes for: refused on the host, where HIP would launch some of
them and say nothing (no GPU needed)."""
import ctypes

import pytest

from test_serving_args import B, FAKE, _cache, _job, _rows  # noqa: F401


@pytest.mark.parametrize("n_rows,n_seq,page", [(1 << 29, 1, 32), ((1 << 31) - 1, 8, 64), (1 << 30, 1 << 23, 1024), ((1 << 27) - 1, 1 << 26, 64)])
def test_pages(B, n_rows, n_seq, page):  # noqa: F811
    L, h, ref = B.lib(), B.Heads(FAKE, 128, 64), ctypes.byref
    c, r = _cache(B, page=page), _rows(B, n_rows=n_rows, n_seq=n_seq)
    for dim in (64, 63):                                     # heads of whole groups of 8 dims, and others
        c.head_dim = dim
        assert L.cmpq_kv_append(ref(c), ref(r), ref(h), ref(h), 0, None, None, None) == -2
        assert L.cmpq_kv_read(ref(c), ref(r), ref(h), ref(h), 0, None, None) == -2


@pytest.mark.parametrize("k", [dict(n_seq=1 << 24, n_rows=1 << 24, max_rows=1, q_heads=2),                     # tiles, few rows
                               dict(n_seq=1, n_rows=(1 << 30) - 513, max_rows=1 << 30, q_heads=2, heads=1),     # tiles, many rows
                               dict(n_seq=1 << 18, n_rows=1 << 20, max_rows=4, q_heads=64, heads=8, max_length=1 << 20),   # joins of either
                               dict(n_seq=1, n_rows=1 << 26, max_rows=1 << 26, q_heads=1, heads=1, max_length=1 << 20)])
def test_attention(B, k):  # noqa: F811
    heads = k.pop("heads", 2)
    job = _job(B, **{"cache": _cache(B, kv_heads=heads, head_dim=8), "ld_table": 1 << 16, **k})
    need = B.lib().cmpq_kv_attention_workspace(ctypes.byref(job))
    assert need > 0 and B.lib().cmpq_kv_attention(ctypes.byref(job), FAKE, need, None) == -2
    assert B.lib().cmpq_kv_attention(ctypes.byref(job), None, 0, None) == -5
