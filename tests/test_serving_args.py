"""The host checks of 8-bit serving: what is refused before anything is launched (no GPU needed)."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2410_13056_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2410_13056_amd import build
        build.build()
    binding.lib()
    return binding


FAKE = 256          # never dereferenced: every call below fails on the host


def test_sizes(B):
    assert B.kv_page_bytes(128, 64) == 64 * 128 and B.kv_page_bytes(80, 32) == 32 * 96 and B.kv_page_bytes(1, 32) == 1024
    for dim, page in ((0, 64), (257, 64), (64, 0), (64, 16), (64, 48), (64, 1056), (-1, 32)):
        assert B.kv_page_bytes(dim, page) == 0
    assert B.int8_weight_bytes(16, 128) == 2048 and B.int8_weight_bytes(17, 129) == 2 * 4 * 1024
    assert B.int8_weight_bytes(4, 131073) == 0 and B.int8_weight_bytes(1 << 24, 4) == 0 and B.int8_weight_bytes(-1, 4) == 0
    n = B.workspace_bytes(B.OP_INT8_PRODUCT, 300, 100, 33)
    assert n % 256 == 0 and n >= 48 * 384 + 33 * 4
    assert B.workspace_bytes(B.OP_INT8_PRODUCT, 1, 1, 0) >= 256


def test_products(B):
    L, ws = B.lib(), 1 << 30
    prep = lambda W=FAKE, dt=0, o=8, i=8, ld=8, c=FAKE, s=FAKE: L.cmpq_int8_prepare(W, dt, o, i, ld, c, s, None, None)
    assert prep(W=None) == prep(c=None) == prep(s=None) == prep(dt=3) == prep(o=-1) == prep(c=FAKE + 8) == -1
    assert prep(ld=7) == prep(i=131073, ld=131073) == prep(o=1 << 24) == -2
    assert prep(o=0) == 0

    def mul(X=FAKE, dt=0, m=4, i=8, ldx=8, c=FAKE, s=FAKE, o=8, Y=FAKE, yd=1, ldy=8, w=FAKE, n=ws):
        return L.cmpq_int8_product(X, dt, m, i, ldx, c, s, o, Y, yd, ldy, w, n, None, None)
    assert mul(X=None) == mul(c=None) == mul(s=None) == mul(Y=None) == mul(dt=3) == mul(yd=-1) == mul(m=-1) == mul(i=0) == -1
    assert mul(ldx=7) == mul(ldy=7) == mul(i=131073, ldx=131073) == mul(m=1 << 24) == -2
    assert mul(w=None) == mul(w=FAKE + 16) == mul(n=256) == -5
    assert mul(m=0) == mul(o=0) == 0


def _cache(B, **k):
    return B.KvCacheView(**{"k_codes": FAKE, "v_codes": FAKE, "k_scale": FAKE, "v_scale": FAKE, "n_pages": 4, "kv_heads": 2,
                            "head_dim": 64, "page": 32, **k})


def _rows(B, **k):
    return B.KvRows(**{"page_table": FAKE, "ld_table": 2, "first": FAKE, "cu_rows": FAKE, "n_seq": 2, "n_rows": 3, **k})


def test_cache_calls(B):
    L, h, ref = B.lib(), B.Heads(FAKE, 128, 64), ctypes.byref

    def append(c=None, r=None, dt=0, K=h, rot=None):
        return L.cmpq_kv_append(ref(c or _cache(B)), ref(r or _rows(B)), ref(K), ref(h), dt, ref(rot) if rot else None, None, None)

    def read(c=None, r=None, dt=0, K=h):
        return L.cmpq_kv_read(ref(c or _cache(B)), ref(r or _rows(B)), ref(K), ref(h), dt, None, None)
    for call in (append, read):
        for bad in (dict(k_codes=None), dict(v_codes=None), dict(k_scale=None), dict(v_scale=None), dict(kv_heads=0), dict(n_pages=-1),
                    dict(k_codes=FAKE + 8)):
            assert call(c=_cache(B, **bad)) == -1, bad
        for bad in (dict(head_dim=0), dict(head_dim=257), dict(page=48), dict(page=2048), dict(kv_heads=70000), dict(n_pages=1 << 31)):
            assert call(c=_cache(B, **bad)) == -2, bad
        for bad in (dict(page_table=None), dict(first=None), dict(cu_rows=None), dict(n_seq=-1), dict(n_rows=-1), dict(ld_table=-1)):
            assert call(r=_rows(B, **bad)) == -1, bad
        assert call(r=_rows(B, n_rows=1 << 31)) == call(r=_rows(B, n_seq=1 << 31)) == -2
        assert call(dt=5) == call(K=B.Heads(None, 1, 1)) == -1
        assert call(r=_rows(B, n_seq=0)) == call(r=_rows(B, n_rows=0)) == call(r=_rows(B, ld_table=0)) == 0
    assert append(rot=B.RotationView(FAKE, None, 8, 64, 0)) == append(rot=B.RotationView(FAKE, FAKE, 0, 64, 0)) == -1
    assert append(rot=B.RotationView(FAKE, FAKE, 8, 63, 0)) == -1 and append(rot=B.RotationView(FAKE, FAKE, 8, 66, 0)) == -2
    assert L.cmpq_kv_append(None, None, None, None, 0, None, None, None) == L.cmpq_kv_read(None, None, None, None, 0, None, None) == -1


def _job(B, **k):
    d = {"cache": _cache(B), "page_table": FAKE, "ld_table": 2, "lengths": FAKE, "cu_rows": FAKE, "n_seq": 2, "n_rows": 3, "max_rows": 2,
         "max_length": 64, "Q": B.Heads(FAKE, 256, 64), "O": B.Heads(FAKE, 256, 64), "q_dtype": 0, "o_dtype": 0, "q_heads": 4,
         "softmax_scale": 0.125, "causal": 1, "window": 0}
    return B.KvAttentionJob(**{**d, **k})


def test_attention(B):
    L, ref = B.lib(), ctypes.byref
    run = lambda ws=FAKE, n=1 << 40, **k: L.cmpq_kv_attention(ref(_job(B, **k)), ws, n, None)
    for bad in (dict(page_table=None), dict(lengths=None), dict(cu_rows=None), dict(Q=B.Heads(None, 1, 1)), dict(O=B.Heads(None, 1, 1)),
                dict(n_seq=-1), dict(n_rows=-1), dict(max_rows=-1), dict(max_length=-1), dict(window=-1), dict(q_dtype=3), dict(o_dtype=1),
                dict(o_dtype=3), dict(q_heads=0), dict(q_heads=5), dict(cache=_cache(B, k_codes=None)), dict(ld_table=-1),
                dict(rotation=B.RotationView(FAKE, None, 8, 64, 0))):
        assert run(**bad) == -1, bad
    for bad in (dict(n_rows=1 << 31), dict(max_length=1 << 31), dict(cache=_cache(B, page=40)),
                dict(rotation=B.RotationView(FAKE, FAKE, 8, 66, 0)), dict(q_heads=1 << 17)):
        assert run(**bad) == -2, bad
    assert run(ws=None) == run(ws=FAKE + 64) == run(n=0) == -5
    assert run(n_seq=0) == run(n_rows=0) == run(max_rows=0) == 0
    assert L.cmpq_kv_attention(None, FAKE, 1 << 40, None) == -1 and L.cmpq_kv_attention_workspace(None) == 0
    size = lambda **k: L.cmpq_kv_attention_workspace(ref(_job(B, **k)))
    assert size() % 256 == 0 and size() >= 256 and size(max_length=1 << 20, ld_table=1 << 15) > size()
