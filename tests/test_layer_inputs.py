"""What blocks hand the layers that share an input.  On the CPU, with the library's part left out."""
import pytest
import torch

from test_feed_forward_args import B, S, _Workspace, _weight  # noqa: F401


@pytest.fixture
def called(B, monkeypatch, S):  # noqa: F811
    """The library's calls, by name."""
    names, lib = [], B._lib

    class Library:
        def __getattr__(self, name):
            f = getattr(lib, name)

            def call(*args):
                names.append(name[5:])
                return f(*args)
            return call
    monkeypatch.setattr(B, "_lib", Library())
    return names


def test_gated_layers_in_8_bits_share_one_coding(S, B, called):  # noqa: F811
    X, down = torch.zeros((5, 64), dtype=torch.bfloat16), _weight(S, B, 24, 64)
    layers = S.GatedLayers(_weight(S, B), _weight(S, B))
    del called[:]
    S.feed_forward_block(X, S.RmsNorm(), layers, down, _Workspace(), add=X)
    assert [n for n in called if not n.endswith("bytes")] == ["rms_norm", "int8_product_job", "int8_product_job", "epilogue", "int8_product_job"]
