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


@pytest.mark.parametrize("kinds", ["fd8", "df8", "8df", "f8d"])
@pytest.mark.parametrize("dtype", TYPES)
def test_layers_of_several_kinds_take_their_own_norms(S, kinds, dtype):  # noqa: F811
    """Functions that of X's type, layers in mixed precision and those in 8 bits beside them that in float16, of one sum."""
    part = Part(S, kinds)
    W = {n: w.to(dtype) for n, w in part.W.items()}
    function = lambda n: lambda x: torch.nn.functional.linear(x, W[n])             # of one type alone
    gate, up = (function(n) if k == "f" else l for n, k, l in zip(("gate", "up"), kinds, (part.gate_up.gate, part.gate_up.up)))
    part.gate_up = S.GatedLayers(gate, up)
    half = torch.float16 if "d" in kinds[:2] else dtype
    for m in (1, 5, 40):
        X, A = _randn(m, m, HIDDEN, dtype=dtype, scale=2), _randn(m + 1, m, HIDDEN)
        for add in (None, A):
            got = part(X, add=add)
            N, stream = (S.rms_norm(X, part.norm.weight, EPS), X) if add is None else S.rms_norm(X, part.norm.weight, EPS, add=add)
            N16 = S.rms_norm(X, part.norm.weight, EPS, add=add, out_dtype=half)
            N16 = N16 if add is None else N16[0]
            G, U = (l(N) if k == "f" else S.apply_layer(l, N16, part.ws) for k, l in zip(kinds, (gate, up)))
            H = S.epilogue(G, activation="silu", times=U, out_dtype=torch.float16 if kinds[2] == "d" else dtype)
            want = S.int8_product(part.down, H, part.ws, out_dtype=dtype, residual=stream) if kinds[2] == "8" else \
                S.epilogue(S.apply_layer(part.down, H, part.ws), residual=stream, out_dtype=dtype)
            assert got.dtype == dtype and torch.equal(got, want) and part.status.item() == 0


@pytest.mark.parametrize("kinds", ["ddd", "dd8", "g8"])
def test_threads_share_layers(S, kinds):  # noqa: F811
    """Two threads in blocks of the same layers, each with its stream and workspace: what each gets alone."""
    import threading
    from paper_2410_13056_amd import binding as B
    part = Part(S, kinds)
    X = [_randn(i, m, HIDDEN, dtype=torch.float16, scale=2) for i, m in ((1, 3), (2, 20))]
    want = [part(x) for x in X]
    got, errors = [[], []], []

    def run(i):
        try:
            ws, stream = B.Workspace(DEV), torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(60):
                    got[i].append(S.feed_forward_block(X[i], part.norm, part.gate_up, part.down, ws))
            stream.synchronize()
        except Exception as e:
            errors.append(e)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in (0, 1)]
    [t.start() for t in threads]
    [t.join(60) for t in threads]
    torch.cuda.synchronize()
    assert not errors
    for i in (0, 1):
        assert len(got[i]) == 60 and all(torch.equal(y, want[i]) for y in got[i])
