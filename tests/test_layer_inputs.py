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


class _Ready:
    """A workspace that has room."""
    buf = torch.empty(0, dtype=torch.uint8)

    def get(self, nbytes):
        return self.buf


def _mixed(d_in, d_out):
    from test_gated_layers_objects import _deployed
    return _deployed(d_in, d_out)


class Linear:
    """A function that takes one type alone, as torch's linear layers do, and gives what the other layers give."""

    def __init__(self, d_in, d_out, dtype):
        self.W, self.seen = torch.ones((d_out, d_in), dtype=dtype), []

    def __call__(self, x):
        self.seen.append(x.dtype)
        return torch.nn.functional.linear(x, self.W).float()


TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("others", ["dd", "d8", "8d", "88", "f8", "fd"])
def test_functions_take_the_norm_in_the_streams_type(S, B, dtype, others, monkeypatch):  # noqa: F811
    """Beside layers in mixed precision too, which read float16."""
    i32, X = (lambda *v: torch.tensor(v, dtype=torch.int32)), torch.zeros((5, 64), dtype=dtype)
    taken = []
    monkeypatch.setattr(B, "kv_page_bytes", lambda dim, page: 2048)
    monkeypatch.setattr(S.P, "lut_matvec", lambda dep, x, ws: taken.append(x.dtype) or torch.zeros((x.shape[0], dep.d_out)))
    make = lambda k: {"d": lambda: _mixed(64, 64), "8": lambda: _weight(S, B, 64, 64), "f": lambda: Linear(64, 64, dtype)}[k]()
    for place in range(3):
        layers = [make(k) for k in others]
        layers.insert(place, Linear(64, 64, dtype))
        cache = S.make_cache(1, 1, 64, 32, "cpu")
        S.attention_block(cache, X, *layers, Linear(64, 64, torch.bfloat16 if dtype == torch.bfloat16 else torch.float16), i32(0)[None], i32(0),
                          i32(5), i32(0, 5), 5, 5, _Ready(), norm=S.RmsNorm())
        assert all(l.seen == [dtype] for l in layers if isinstance(l, Linear))
    for k in others:
        for pair in ((make(k), Linear(64, 64, dtype)), (Linear(64, 64, dtype), make(k))):
            for add in (None, X.float()):
                S.feed_forward_block(X, S.RmsNorm(), S.GatedLayers(*pair), make(others[0]), _Ready(), add=add)
            assert all(set(l.seen) == {dtype} for l in pair if isinstance(l, Linear))
    assert set(taken) <= {torch.float16}
