"""A decoder layer's feed-forward part, its operators together, and the whole layer with its attention."""
import numpy as np
import pytest
import torch

import feed_forward_reference as Q
import serving_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
HIDDEN, FF = 256, 700
TYPES = [torch.float16, torch.bfloat16, torch.float32]
EPS = 1e-5


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _randn(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * scale).to(dtype)


class Part:
    """Projections of either kind: "8" 8-bit integers, "g" gate and second factor as one, "f" a function, "d" mixed precision."""

    def __init__(self, S, kinds, ff=FF):
        from paper_2410_13056_amd import binding as B
        self.S, self.ws, self.status = S, B.Workspace(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        self.W = {n: _randn(i, o, d, dtype=torch.float16, scale=d ** -0.5) for i, (n, o, d) in
                  enumerate((("gate", ff, HIDDEN), ("up", ff, HIDDEN), ("down", HIDDEN, ff)))}
        self.norm = S.RmsNorm(1 + 0.2 * _randn(9, HIDDEN), EPS)
        self.down = self.layer("down", kinds[-1])
        self.gate_up = S.prepare_int8_gated(self.W["gate"], self.W["up"]) if kinds[0] == "g" else \
            S.GatedLayers(self.layer("gate", kinds[0]), self.layer("up", kinds[1]))

    def layer(self, name, kind):
        W = self.W[name]
        if kind == "8":
            return self.S.prepare_int8(W)
        if kind == "f":
            return lambda x: x.float() @ W.float().t()
        from paper_2410_13056_amd import pipeline as P
        _, sumsq = P.activation_stats(_randn(5, 512, W.shape[1], dtype=torch.float16), self.ws)
        return P.prepare_deployment(P.quantize_layer(W, sumsq, (2, 3, 4), 3.5, 4500, 10000, 5, self.ws), self.ws)

    def __call__(self, X, **k):
        got = self.S.feed_forward_block(X, self.norm, self.gate_up, self.down, self.ws, status=self.status, **k)
        torch.cuda.synchronize()
        return got


@pytest.mark.parametrize("m", [1, 2, 7, 40, 600])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
def test_all_in_8_bits(S, m, dtype, act):
    """Against 64 bits from the hidden values on.  Those are checked on their own; the output's sums are exact, so what is off is
    their scaling and the roundings behind it."""
    part = Part(S, "g8")
    X, A = _randn(m, m, HIDDEN, dtype=dtype, scale=2), _randn(m + 1, m, HIDDEN)
    for add in (None, A):
        got = part(X, add=add, activation=act)
        assert got.dtype == dtype and part.status.item() == 0
        y, s = Q.norm(X, add, part.norm.weight, EPS, dtype)
        rows = S.rms_norm(X, part.norm.weight, EPS, add=add, coded=True)
        rows = rows if add is None else rows[0]
        assert np.array_equal(Q.coded(rows)[0], R.rows_in_8_bits(y)[0])
        H = S.int8_gated_product(part.gate_up, rows, part.ws, act, out_dtype=dtype)
        (g, eg), (u, eu) = (Q.product(torch.from_numpy(y), part.W[n]) for n in ("gate", "up"))
        want, bound = Q.finish(g, eg, None, act, u, eu)
        Q.check(H, want, bound)
        want, bound = Q.finish(*Q.product(H, part.W["down"]), residual=Q.f64(s))
        Q.check(got, want, bound)


@pytest.mark.parametrize("kinds", ["fff", "88f", "8f8", "g8", "gf", "gd", "dd8", "ddd", "ddf", "d8d", "fd8"])
@pytest.mark.parametrize("dtype", TYPES)
def test_kinds_of_layers(S, kinds, dtype):
    """Against the same layers one by one, what stands between them in 64 bits.  Apart from what both sides have: the norm and the
    hidden values rounded to 16 bits (2^-8 each in bfloat16; a code may flip, 2^-7 of the largest of a row, of some rows), sums of
    700 products of independent roundings: 2^-6 in all of the branch's norm."""
    part = Part(S, kinds)
    for m in (1, 3, 50):
        X, A = _randn(m, m, HIDDEN, dtype=dtype, scale=2), _randn(m + 1, m, HIDDEN)
        got = part(X, add=A)
        assert got.dtype == dtype and part.status.item() == 0
        y, s = Q.norm(X, A, part.norm.weight, EPS, dtype)
        N = torch.from_numpy(y).to(DEV)
        if kinds[0] == "g":
            G, U = (S.int8_product(S.prepare_int8(part.W[n]), N, part.ws, out_dtype=torch.float32) for n in ("gate", "up"))
        else:
            G, U = (S.apply_layer(l, N, part.ws) for l in (part.gate_up.gate, part.gate_up.up))
        H = torch.nn.functional.silu(G.double()) * U.double()
        D = S.apply_layer(part.down, H.float(), part.ws).double().cpu()
        branch = got.double().cpu() - s.double()
        room = 2.0 ** -6 * D.norm() + Q.ROUND[dtype] * got.double().cpu().norm()
        assert (branch - D).norm() <= room, ((branch - D).norm() / D.norm(), room)


def test_layers_whose_outputs_are_views_and_no_rows(S):
    part, plain = Part(S, "fff"), Part(S, "fff")
    X = _randn(1, 9, HIDDEN, dtype=torch.float16)
    part.gate_up = S.GatedLayers(lambda x: plain.gate_up.gate(x).t().contiguous().t(), lambda x: plain.gate_up.up(x).repeat(1, 2)[:, :FF])
    part.down = lambda x: plain.down(x).t().contiguous().t()
    assert torch.equal(part(X), plain(X))
    for kinds in ("fff", "g8", "ddd"):
        assert Part(S, kinds)(torch.empty((0, HIDDEN), device=DEV).half()).shape == (0, HIDDEN)


@pytest.mark.parametrize("kinds", ["g8", "ddd", "f8f"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_inputs_that_are_no_finite_numbers_are_flagged_and_stay_in_their_rows(S, kinds, value):
    from paper_2410_13056_amd import binding as B
    part = Part(S, kinds)
    X = _randn(1, 20, HIDDEN, dtype=torch.float16)
    want = part(X)
    assert part.status.item() == 0
    X[3, 100] = value
    got = part(X)
    assert part.status.item() & B.STATUS_NONFINITE
    others = torch.arange(20, device=DEV) != 3
    assert torch.equal(got[others], want[others])


def test_a_graph_of_the_block(S):
    for kinds, m in (("g8", 1), ("g8", 30), ("ddd", 2)):
        part = Part(S, kinds)
        X = _randn(1, m, HIDDEN, dtype=torch.bfloat16)
        part(X)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = S.feed_forward_block(X, part.norm, part.gate_up, part.down, part.ws)
        for k in range(3):
            X.copy_(_randn(10 + k, m, HIDDEN))
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            assert torch.equal(got, part(X))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_decoder_layer(S, dtype):
    """Attention and feed-forward part of a layer one after the other, for a prompt and single tokens, all in 8 bits: against
    the operators called one by one, bit for bit."""
    heads, kv, dim, page = 8, 2, 32, 32
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    part = Part(S, "g8")
    layers = [S.prepare_int8(_randn(20 + i, o, d, dtype=torch.float16, scale=d ** -0.5)) for i, (o, d) in
              enumerate(((heads * dim, HIDDEN), (kv * dim, HIDDEN), (kv * dim, HIDDEN), (HIDDEN, heads * dim)))]
    norm, rot = S.RmsNorm(1 + 0.1 * _randn(8, HIDDEN), EPS), S.make_rotation(100, dim, device=DEV)
    caches, held = [S.make_cache(4, kv, dim, page, DEV) for _ in range(2)], 0
    for n in (45, 1, 1, 4):
        X = _randn(n, n, HIDDEN, dtype=dtype)
        where = (i32([[2, 0, 3]]), i32([held]), i32([held + n]), i32([0, n]), n, held + n, part.ws, rot)
        A = S.attention_block(caches[0], X, *layers, *where, status=part.status, norm=norm)
        got = part(X, add=A)
        rows = S.rms_norm(X, norm.weight, norm.eps, coded=True)
        again = S.attention_block(caches[1], X, *[lambda x, l=l: S.int8_product(l, rows, part.ws, out_dtype=torch.float32) for l in layers[:3]],
                                  lambda o: S.int8_product(layers[3], o, part.ws, out_dtype=torch.float32), *where,
                                  attention_dtype=torch.bfloat16 if dtype == torch.bfloat16 else torch.float16)
        assert torch.equal(A, again) and part.status.item() == 0
        s = X.float() + A.float()
        stream = s.to(dtype)
        coded = S.rms_norm(stream, part.norm.weight, EPS, coded=True)
        H = S.int8_gated_product(part.gate_up, coded, part.ws, out_dtype=dtype)
        assert torch.equal(got, S.int8_product(part.down, H, part.ws, out_dtype=dtype, residual=stream))
        held += n


def test_attention_of_a_normed_stream_with_layers_of_different_kinds(S):
    """With a norm, layers that are not all in 8 bits read its values."""
    heads, kv, dim = 8, 2, 32
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    from paper_2410_13056_amd import binding as B
    ws, norm = B.Workspace(DEV), S.RmsNorm(None, EPS)
    W = [_randn(20 + i, o, d, dtype=torch.float16, scale=d ** -0.5) for i, (o, d) in
         enumerate(((heads * dim, HIDDEN), (kv * dim, HIDDEN), (kv * dim, HIDDEN), (HIDDEN, heads * dim)))]
    layers = [lambda x: x.float() @ W[0].float().t(), S.prepare_int8(W[1]), S.prepare_int8(W[2]), S.prepare_int8(W[3])]
    X = _randn(1, 12, HIDDEN, dtype=torch.bfloat16)
    where = (i32([[0]]), i32([0]), i32([12]), i32([0, 12]), 12, 12, ws)
    got = S.attention_block(S.make_cache(1, kv, dim, 32, DEV), X, *layers, *where, norm=norm)
    N = S.rms_norm(X, None, EPS)
    assert torch.equal(got, S.attention_block(S.make_cache(1, kv, dim, 32, DEV), N, *layers, *where))


@pytest.mark.parametrize("n", [1, 2, 3, 40])
def test_attention_codes_its_input_once(S, n):
    """Three layers in 8 bits read rows coded once: what each would make of the values by itself, bit for bit."""
    heads, kv, dim = 8, 2, 32
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    from paper_2410_13056_amd import binding as B
    ws, status = B.Workspace(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    W = [_randn(20 + i, o, d, dtype=torch.float16, scale=d ** -0.5) for i, (o, d) in
         enumerate(((heads * dim, HIDDEN), (kv * dim, HIDDEN), (kv * dim, HIDDEN), (HIDDEN, heads * dim)))]
    layers = [S.prepare_int8(w) for w in W]
    X = _randn(1, n, HIDDEN + 3, dtype=torch.bfloat16)[:, 1:1 + HIDDEN]
    where = (i32([[0, 1]]), i32([0]), i32([n]), i32([0, n]), n, n, ws)
    got = S.attention_block(S.make_cache(2, kv, dim, 32, DEV), X, *layers, *where, status=status)
    each = [lambda x, l=l: S.int8_product(l, x, ws, out_dtype=torch.float32) for l in layers[:3]]
    assert torch.equal(got, S.attention_block(S.make_cache(2, kv, dim, 32, DEV), X, *each, layers[3], *where))
    assert status.item() == 0
    X[n - 1, 5] = float("inf")
    S.attention_block(S.make_cache(2, kv, dim, 32, DEV), X, *layers, *where, status=status)
    assert status.item() == B.STATUS_NONFINITE


@pytest.mark.parametrize("m", [1, 2, 3, 16, 50, 300, 2100])
@pytest.mark.parametrize("dtype", TYPES)
def test_one_call_is_its_three_bit_for_bit(S, m, dtype):
    """Whatever the types of what is added, the weight and the hidden values; rows that lie apart; the answer in the place of the
    stream or of what is added."""
    from paper_2410_13056_amd import binding as B
    part = Part(S, "g8", 1500)
    X, A = (_randn(i, m, HIDDEN + 8, dtype=t)[:, 3:3 + HIDDEN] for i, t in ((1, dtype), (2, torch.float32)))
    for add, act, hidden in ((None, "silu", None), (A, "gelu", torch.bfloat16), (X, None, torch.float32), (A.half(), "relu", torch.float16)):
        got = part(X, add=add, activation=act, hidden_dtype=hidden)
        rows = S.rms_norm(X, part.norm.weight, EPS, add=add, coded=True)
        rows, stream = (rows, X) if add is None else rows
        H = S.int8_gated_product(part.gate_up, rows, part.ws, act, out_dtype=hidden or dtype)
        assert torch.equal(got, S.int8_product(part.down, H, part.ws, out_dtype=dtype, residual=stream))
        args = (part.norm.weight, EPS, part.gate_up._args, part.down._args)
        for place in [X] if add is None else [X, add]:
            if place.dtype != dtype:
                continue
            whole = {id(t): (t if t._base is None else t._base).clone() for t in (X, add) if t is not None}
            mine = {k: w if w.shape[1] == HIDDEN else w[:, 3:3 + HIDDEN] for k, w in whole.items()}
            Y = mine[id(place)]
            B.int8_feed_forward(mine[id(X)], *args, Y, part.ws, None if add is None else mine[id(add)], act, hidden)
            assert torch.equal(Y, got)
            if place._base is not None:
                assert torch.equal(whole[id(place)][:, -5:], place._base[:, -5:]) and torch.equal(whole[id(place)][:, :3], place._base[:, :3])
