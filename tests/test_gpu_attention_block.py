"""A decoder layer's attention, its operators together: what goes wrong in one shows, whatever kinds the layers are."""
import pytest
import torch

import serving_reference as R  # noqa: F401  (the folder of the tests is on the path)

pytestmark = pytest.mark.gpu

DEV = "cuda"
HIDDEN, HEADS, KV, DIM, PAGE = 256, 8, 2, 32, 32


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Block:
    """Layers of either kind, a cache of two sequences; `step` runs the block for new rows of each."""

    def __init__(self, S, kinds="8888", seed=0):
        from paper_2410_13056_amd import binding as B
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.S, self.ws = S, B.Workspace(DEV)
        self.W = {n: torch.randn((o, i), generator=g, device=DEV).half() * i ** -0.5 for n, o, i in
                  (("q", HEADS * DIM, HIDDEN), ("k", KV * DIM, HIDDEN), ("v", KV * DIM, HIDDEN), ("o", HIDDEN, HEADS * DIM))}
        self.layers = {n: S.prepare_int8(w) if kind == "8" else (lambda x, w=w: x.float() @ w.float().t())
                       for (n, w), kind in zip(self.W.items(), kinds)}
        self.cache, self.rot = S.make_cache(8, KV, DIM, PAGE, DEV), S.make_rotation(100, DIM, device=DEV)
        self.table, self.held = _i32([[5, 1, 0], [2, 7, 3]]), [0, 0]
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step(self, X, new, **kw):
        lens, cu = [h + n for h, n in zip(self.held, new)], _i32([0, new[0], sum(new)])
        L = self.layers
        out = self.S.attention_block(self.cache, X, L["q"], L["k"], L["v"], L["o"], self.table, _i32(self.held), _i32(lens), cu,
                                     max(new), max(lens), self.ws, self.rot, status=self.status, **kw)
        torch.cuda.synchronize()
        self.held = lens
        return out


@pytest.mark.parametrize("kinds", ["8888", "8fff", "f8ff", "ff8f", "fff8"])
@pytest.mark.parametrize("new", [[1, 1], [20, 40]])
@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
def test_inputs_that_are_no_finite_numbers_are_flagged(S, kinds, new, value):
    from paper_2410_13056_amd import binding as B
    b = Block(S, kinds)
    X = torch.randn((sum(new), HIDDEN), device=DEV).half()
    b.step(X, new)
    assert b.status.item() == 0
    X[0, 3] = value
    b.step(X[:2], [1, 1])
    assert b.status.item() == B.STATUS_NONFINITE


@pytest.mark.parametrize("kinds", ["ffff", "fff8", "8888"])
def test_values_beyond_float16_of_a_bfloat16_model(S, kinds):
    """Values of some millions: finite, and right.  Rounded: X's codes not at all (the same codes on both sides), the attention's
    output to bfloat16 (2^-9 of itself, and once more as 8-bit codes of the largest of a row where `o` has them, 2^-8 of the
    largest, at most 4 times the row's norm / sqrt(256)), its weights to FP16."""
    import numpy as np
    b = Block(S, "ffff")
    b.W["v"] *= 0
    b.W["v"] += torch.randn((KV * DIM, HIDDEN), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).half() * 2048
    b.layers = {n: S.prepare_int8(w) if kind == "8" else (lambda x, w=w: x.float() @ w.float().t()) for (n, w), kind in zip(b.W.items(), kinds)}
    new = [30, 12]
    X = torch.randn((42, HIDDEN), generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).bfloat16() * 64
    b.layers["q"] = lambda x: x.float() @ b.W["q"].float().t() / 64
    got = b.step(X, new)
    assert got.isfinite().all() and b.status.item() == 0
    q, want, at = R.as_f32(b.layers["q"](X)).reshape(-1, HEADS, DIM), [], 0
    for i, n in enumerate(new):
        k, v = (t.double().cpu().numpy() for t in S.kv_read(b.cache, b.table[i:i + 1].contiguous(), _i32([0]), _i32([0, n]), n, torch.float32))
        assert np.abs(v).max() > 1e5
        x = R.turn(q[at:at + n], np.arange(n), R.as_f32(b.rot.cos), R.as_f32(b.rot.sin), False)
        want.append(R.attention(x.astype(np.float64), k, v, DIM ** -0.5, True, 0)[0])
        at += n
    want = np.concatenate(want).reshape(42, -1) @ b.W["o"].double().cpu().numpy().T
    rel = np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)
    assert rel <= 2.0 ** -8 + (2.0 ** -6 if kinds[3] == "8" else 0), rel
    b.held = [0, 0]
    half = b.step(X, new, attention_dtype=torch.float16)                # as asked for: infinite
    assert kinds[3] == "8" and b.status.item() or not half.isfinite().all()


@pytest.mark.parametrize("kinds", ["8888", "ffff"])
def test_no_rows_and_layers_whose_outputs_are_views(S, kinds):
    b = Block(S, kinds)
    assert b.step(torch.empty((0, HIDDEN), device=DEV).half(), [0, 0]).shape == (0, HIDDEN)
    X = torch.randn((9, HIDDEN), device=DEV).half()
    want = b.step(X, [4, 5])
    b.held = [0, 0]
    plain = dict(b.layers)
    for n in b.layers:                                                   # rows that lie apart, and columns
        b.layers[n] = lambda x, n=n: S.apply_layer(plain[n], x, b.ws).t().contiguous().t()
    assert torch.equal(b.step(X, [4, 5]), want) and b.status.item() == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("deployed", ["qo", "qkvo"])
def test_layers_in_mixed_precision(S, dtype, deployed):
    """Queries and outputs, or all, through the mixed-precision tables: a prompt and steps, against the same layers one by one.
    Rounded apart from what both sides have: the query to 2^-16 of its row's largest, weights to FP16, the attention's output
    to FP16 (what those layers read): 2^-10 in all."""
    import numpy as np
    from paper_2410_13056_amd import pipeline as P
    b = Block(S, "8888")
    g = torch.Generator(device=DEV).manual_seed(4)
    for n in deployed:
        d_in = b.W[n].shape[1]
        X = torch.randn((512, d_in), generator=g, device=DEV).half()
        _, sumsq = P.activation_stats(torch.randn((512, d_in), generator=g, device=DEV).half(), b.ws)
        r = P.quantize_layer(b.W[n], sumsq, (2, 3, 4), 3.5, 4500, 10000, 5, b.ws)
        b.layers[n] = P.prepare_deployment(r, b.ws)
    for new in ([40, 7], [1, 1], [3, 2]):
        X = torch.randn((sum(new), HIDDEN), generator=g, device=DEV).to(dtype)
        got = b.step(X, new)
        assert b.status.item() == 0
        q, want, at = R.as_f32(S.apply_layer(b.layers["q"], X, b.ws)).reshape(-1, HEADS, DIM), [], 0
        for i, n in enumerate(new):
            t = b.held[i]
            k, v = (x.double().cpu().numpy() for x in S.kv_read(b.cache, b.table[i:i + 1].contiguous(), _i32([0]), _i32([0, t]), t, torch.float32))
            x = R.turn(q[at:at + n], t - n + np.arange(n), R.as_f32(b.rot.cos), R.as_f32(b.rot.sin), False)
            want.append(R.attention(x.astype(np.float64), k, v, DIM ** -0.5, True, 0)[0])
            at += n
        attended = torch.from_numpy(np.concatenate(want)).flatten(1).to(DEV).half()
        ref = S.apply_layer(b.layers["o"], attended, b.ws).double()
        assert ((got.double() - ref).norm() / ref.norm()).item() <= 2.0 ** -10
