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
