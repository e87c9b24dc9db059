"""What layers are handed that share an input: blocks against the operators called one by one, bit for bit."""
import pytest
import torch

from test_gpu_feed_forward_block import DEV, EPS, HIDDEN, Part, S, TYPES, _randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [1, 2, 3, 50, 600])
@pytest.mark.parametrize("dtype", TYPES)
def test_two_gated_layers_in_8_bits_read_rows_coded_once(S, m, dtype):  # noqa: F811
    """From the norm in fp32, as one layer of both does."""
    part, one = Part(S, "888"), Part(S, "g8")
    X, A = _randn(m, m, HIDDEN, dtype=dtype, scale=2), _randn(m + 1, m, HIDDEN)
    for add in (None, A):
        got = part(X, add=add)
        rows = S.rms_norm(X, part.norm.weight, EPS, add=add, coded=True)
        rows, stream = (rows, X) if add is None else rows
        G, U = (S.int8_product(l, rows, part.ws, out_dtype=torch.float32) for l in (part.gate_up.gate, part.gate_up.up))
        H = S.epilogue(G, activation="silu", times=U, out_dtype=dtype)
        assert torch.equal(got, S.int8_product(part.down, H, part.ws, out_dtype=dtype, residual=stream))
        assert torch.equal(got, one(X, add=add)) and part.status.item() == 0
