"""8-bit products without anything behind them, and the coding of rows: what lies on another device than the current one is
refused before its address reaches the library.  On the CPU: nothing here is launched."""
import pytest
import torch

from test_feed_forward_args import B, S, _Workspace, _weight  # noqa: F401


class Elsewhere(torch.Tensor):
    """A host tensor that says that it lies on the next device."""
    def get_device(self):
        return 1


def _elsewhere(t):
    return t.as_subclass(Elsewhere)


class _OtherWorkspace:
    class buf:
        get_device = staticmethod(lambda: 1)


def test_plain_products(S, B):  # noqa: F811
    w, X, flags = _weight(S, B), torch.zeros((3, 64)), torch.zeros(1, dtype=torch.int32)
    out = torch.empty((3, 24))
    assert S.int8_product(w, X, _Workspace(), out=out, status=flags) is out
    for bad in (dict(ws=_OtherWorkspace()), dict(X=_elsewhere(X)), dict(out=_elsewhere(out)), dict(status=_elsewhere(flags))):
        with pytest.raises(ValueError, match="device"):
            S.int8_product(**{**dict(w=w, X=X, ws=_Workspace(), out=out, status=flags), **bad})
    with pytest.raises(ValueError, match="device"):
        S.int8_product(S.Int8Weight(64, 24, _elsewhere(w.codes), w.scale), X, _Workspace(), out=out)
    with pytest.raises(ValueError, match="device"):
        S.apply_layer(w, X, _OtherWorkspace())


def test_coding_of_rows(S, B):  # noqa: F811
    X, flags = torch.zeros((24, 64)), torch.zeros(1, dtype=torch.int32)
    codes, scale = torch.empty(B.int8_weight_bytes(24, 64), dtype=torch.int8), torch.empty(24)
    B.int8_prepare(X, codes, scale, flags)
    for at in range(4):
        args = [X, codes, scale, flags]
        args[at] = _elsewhere(args[at])
        with pytest.raises(ValueError, match="device"):
            B.int8_prepare(*args)
    with pytest.raises(ValueError, match="device"):
        S.int8_rows(_elsewhere(X), out=S.Int8Rows(24, 64, codes, scale))


def test_codes_and_scales_of_two_devices(S, B):  # noqa: F811
    w = _weight(S, B)
    with pytest.raises(ValueError, match="device"):
        S.Int8Weight(64, 24, w.codes, _elsewhere(w.scale))
    with pytest.raises(ValueError, match="device"):
        S.Int8Rows(24, 64, w.codes, _elsewhere(w.scale))
