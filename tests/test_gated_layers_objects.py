"""Layers of a gated feed-forward part that a program keeps and its threads share.  On the CPU: nothing here is launched."""
import threading

import pytest
import torch

from test_serving_objects import S  # noqa: F401


def _deployed(d_in=64, d_out=24):
    """A layer in mixed precision whose channels are all kept whole: the least that a call describes."""
    from paper_2410_13056_amd import pipeline as P
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    return P.Deployed(d_in, d_out, (2, 4), [0, 0], [None, None], [None, None], [None, None], torch.arange(d_in, dtype=torch.int32),
                      torch.zeros((d_in, d_out), dtype=torch.float16), i32(d_out + 1), i32(0), torch.zeros(0))


class _Workspace:
    buf = torch.empty(1, dtype=torch.uint8)

    def get(self, nbytes):
        return self.buf


class _Library:
    """The library without its launches: `called(layers, n)` in place of the products of a group."""

    def __init__(self, real, called):
        self.real, self.called = real, called

    def __getattr__(self, name):
        if name.startswith("cmpq_lut_matvec_group"):
            return lambda arr, n, m, *rest: self.called(arr, n) or 0
        return getattr(self.real, name)


def _pointers(arr, n):
    return [(arr[i].X, arr[i].ldx, arr[i].Y, arr[i].ldy) for i in range(n)]


def test_threads_in_one_pair_of_layers_have_their_own_arguments(S, monkeypatch):  # noqa: F811
    """Two threads are in the library at once; each call reads its arguments when both have been handed theirs."""
    from paper_2410_13056_amd import binding as B
    meet, seen, errors = threading.Barrier(2), {}, []

    def called(arr, n):
        meet.wait(20)
        seen[threading.get_ident()] = _pointers(arr, n)
        meet.wait(20)
    monkeypatch.setattr(B, "_lib", _Library(B.lib(), called))
    layers, want = S.GatedLayers(_deployed(), _deployed()), {}

    def run(rows):
        try:
            X = torch.zeros((rows, 64), dtype=torch.float16)
            Y = layers.apply(X, _Workspace())
            want[threading.get_ident()] = [(X.data_ptr(), 64, y.data_ptr(), 24) for y in Y]
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=run, args=(n,)) for n in (3, 5)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and len(seen) == 2 and seen == want


def test_calls_one_after_the_other_and_refused_ones(S, monkeypatch):  # noqa: F811
    """A group's calls describe their own tensors, also after one that was refused half way."""
    from paper_2410_13056_amd import binding as B, pipeline as P
    seen = []
    monkeypatch.setattr(B, "_lib", _Library(B.lib(), lambda arr, n: seen.append((_pointers(arr, n), [arr[i].d_out for i in range(n)]))))
    group = P.group_products([_deployed(64, 24), _deployed(64, 16)])
    for rows in (1, 4, 2):
        X = torch.zeros((rows, 70), dtype=torch.float16)[:, 3:67]
        Y = [torch.empty((rows, n)) for n in (24, 16)]
        with pytest.raises(ValueError):
            group([X, X[:, :60]], Y, _Workspace())
        group([X, X], Y, _Workspace())
        assert seen.pop() == ([(X.data_ptr(), 70 if rows > 1 else 64, y.data_ptr(), y.shape[1]) for y in Y], [24, 16]) and not seen


def test_copies_are_copies(S):  # noqa: F811
    import copy
    import pickle
    layers = S.GatedLayers(_deployed(), _deployed())
    for other in (copy.deepcopy(layers), pickle.loads(pickle.dumps(layers))):
        for a, b in ((layers.gate, other.gate), (layers.up, other.up)):
            assert torch.equal(a.act_idx, b.act_idx) and a.act_idx.data_ptr() != b.act_idx.data_ptr()
            assert b.call() is not a.call() and b.call()._head[7] == b.act_idx.data_ptr()
        assert other._args is not layers._args and other._args._arr[1].act_idx == other.up.act_idx.data_ptr()
    shallow = copy.copy(layers)
    assert shallow.gate is layers.gate and shallow._args is not layers._args
    one = copy.copy(layers.gate)
    one.act_idx = one.act_idx.clone()                        # a copy's calls read what its fields say
    assert one.call()._head[7] == one.act_idx.data_ptr() != layers.gate.call()._head[7]
