"""The objects that a program of 8-bit serving keeps - caches, rotations, layers: what they hold on to and what a call is
handed.  On the CPU: nothing here is launched."""
import gc
import weakref

import pytest
import torch


@pytest.fixture
def S(monkeypatch):
    import os
    from paper_2410_13056_amd import binding, serving
    if not os.path.exists(binding.LIB_PATH):
        from paper_2410_13056_amd import build
        build.build()
    binding.lib()
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else t.data_ptr())
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    return serving


def _weight(S, d_in=64, d_out=16):
    from paper_2410_13056_amd import binding as B
    return S.Int8Weight(d_in, d_out, torch.zeros(B.int8_weight_bytes(d_out, d_in), dtype=torch.int8), torch.ones(d_out))


def test_dropped_objects_give_their_memory_back(S):
    for make, names in ((lambda: S.make_cache(2, 2, 64, 32, "cpu"), ("k", "v", "k_scale", "v_scale")),
                        (lambda: S.make_rotation(8, 64, device="cpu"), ("cos", "sin")), (lambda: _weight(S), ("codes", "scale"))):
        thing = make()
        held = [weakref.ref(getattr(thing, n)) for n in names]
        del thing
        gc.collect()
        assert [r() for r in held] == [None] * len(held), names


def _calls(S, cache, n):
    """Append, read and attention with n rows."""
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    x, table, zero, cu = torch.zeros((n, 2, 64)), torch.zeros((1, n), dtype=torch.int32), i32(0), i32(0, n)
    return {"append": lambda: S.kv_append(cache, x, x, table, zero, cu),
            "read": lambda: S.kv_read(cache, table, zero, cu, n, torch.float32),
            "attention": lambda: S.kv_attention(cache, x, table, zero, cu, n, n, ws=_NoWorkspace())}


class _NoWorkspace:
    buf = torch.empty(0, dtype=torch.uint8)


@pytest.mark.parametrize("kind", ["append", "read", "attention"])
def test_threads_in_calls_on_one_cache_have_their_own_arguments(S, monkeypatch, kind):
    """Two threads are in the library at once; each of its two calls reads its arguments when both have been handed them."""
    import threading
    from paper_2410_13056_amd import binding as B
    meet, seen = threading.Barrier(2), {}

    class Library:
        def __getattr__(self, name):
            def call(*args):
                meet.wait(20)
                got = args[0] if name == "cmpq_kv_attention" else args[1]
                got = getattr(got, "_obj", got)
                seen[threading.get_ident()] = (got.n_rows, got.ld_table)
                meet.wait(20)
                return 0
            return call

    cache, want, errors = S.make_cache(8, 2, 64, 32, "cpu"), {}, []
    monkeypatch.setattr(B, "_lib", Library())

    def run(n):
        want[threading.get_ident()] = (n, n)
        try:
            _calls(S, cache, n)[kind]()
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=run, args=(n,)) for n in (3, 5)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and seen == want


def test_assigned_fields_are_what_the_next_call_takes(S):
    cache = S.make_cache(4, 2, 64, 32, "cpu")
    names = {"k": "k_codes", "v": "v_codes", "k_scale": "k_scale", "v_scale": "v_scale"}
    for name, field in names.items():
        t = getattr(cache, name).clone()
        setattr(cache, name, t)
        assert getattr(cache._view, field) == t.data_ptr()
    cache.k = cache.k[:3].contiguous()                                   # no cache any more
    with pytest.raises(ValueError):
        cache._view
    weight = _weight(S)
    weight.scale = weight.scale.clone()
    assert weight._args._scale == weight.scale.data_ptr()
    rotation = S.make_rotation(8, 64, device="cpu")
    rotation.cos, rotation.sin = rotation.cos[:5].contiguous(), rotation.sin[:5].contiguous()
    assert rotation._args.positions == 5 and rotation._args.cos == rotation.cos.data_ptr()


def test_copies_are_copies(S, tmp_path):
    import copy
    import pickle
    for thing, names in ((S.make_cache(2, 2, 64, 32, "cpu"), ("k", "v", "k_scale", "v_scale")),
                         (S.make_rotation(8, 64, device="cpu"), ("cos", "sin")), (_weight(S), ("codes", "scale"))):
        for other in (copy.deepcopy(thing), pickle.loads(pickle.dumps(thing))):
            assert type(other) is type(thing) and other._args is not thing._args
            for n in names:
                a, b = getattr(thing, n), getattr(other, n)
                assert torch.equal(a.nan_to_num(), b.nan_to_num()) and a.data_ptr() != b.data_ptr()
        shallow = copy.copy(thing)
        assert all(getattr(shallow, n) is getattr(thing, n) for n in names) and shallow._args is not thing._args


def test_rotations_of_dims_that_are_no_pairs_are_refused(S):
    for positions, dims in ((8, 7), (8, 1), (8, 0), (8, -2), (0, 64)):
        with pytest.raises(ValueError):
            S.make_rotation(positions, dims, device="cpu")
    assert S.make_rotation(1, 2, device="cpu").cos.shape == (1, 1)


def test_objects_that_calls_were_made_with_give_their_memory_back(S, monkeypatch):
    from paper_2410_13056_amd import binding as B
    monkeypatch.setattr(B, "_lib", type("Library", (), {"__getattr__": lambda self, name: lambda *args: 0})())
    real = S.make_cache
    monkeypatch.setattr(B, "kv_page_bytes", lambda dim, page: 2048)
    cache, rotation = real(8, 2, 64, 32, "cpu"), S.make_rotation(8, 64, device="cpu")
    held = [weakref.ref(t) for t in (cache.k, cache.v_scale, rotation.cos)]
    for n in (1, 2):
        for call in _calls(S, cache, n).values():
            call()
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    x = torch.zeros((1, 2, 64))
    S.kv_append(cache, x, x, i32(0)[None], i32(0), i32(0, 1), rotation)
    S.kv_attention(cache, x, i32(0)[None], i32(1), i32(0, 1), 1, 1, ws=_NoWorkspace(), rotation=rotation)
    with pytest.raises(ValueError):
        S.kv_append(cache, x[:, :1], x, i32(0)[None], i32(0), i32(0, 1))
    del cache, rotation, call
    gc.collect()
    assert [r() for r in held] == [None] * 3
