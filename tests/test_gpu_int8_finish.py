"""Products in 8-bit integers with what follows them, and gated ones, through the public calls: the sums are exact, so the
outputs are held to 64 bits within the roundings of the steps behind them."""
import numpy as np
import pytest
import torch

import feed_forward_reference as Q
import serving_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _randn(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * scale).to(dtype)


def _ws():
    from paper_2410_13056_amd import binding as B
    return B.Workspace(DEV)


def _product(S, X, W, w=None, p=None, rows=False, **k):
    want, bound = Q.finish(*(p or Q.product(X, W)), Q.f64(k.get("bias")), k.get("activation"), residual=Q.f64(k.get("residual")))
    got = S.int8_product(w or S.prepare_int8(W), S.int8_rows(X) if rows else X, _ws(), **k)
    torch.cuda.synchronize()
    Q.check(got, want, bound)
    return got


def _gated(S, X, Wg, Wu, w=None, p=None, rows=False, **k):
    (g, eg), (u, eu) = p or (Q.product(X, Wg), Q.product(X, Wu))
    want, bound = Q.finish(g, eg, Q.f64(k.get("gate_bias")), k.get("activation", "silu"), u, eu, Q.f64(k.get("up_bias")), Q.f64(k.get("residual")))
    got = S.int8_gated_product(w or S.prepare_int8_gated(Wg, Wu), S.int8_rows(X) if rows else X, _ws(), **k)
    torch.cuda.synchronize()
    Q.check(got, want, bound)
    return got


# between them every kernel, with edges that are part full: one launch; 2 and 1 pieces by 8 and 16 wavefronts; 4 x 2 pieces; the
# four sizes of tiles
SIZES = [(1, 1, 1), (1, 64, 16), (2, 127, 70), (1, 4096, 1000), (1, 16384, 50), (1, 16385, 40), (2, 16400, 64), (2, 63, 17), (3, 1030, 515),
         (5, 129, 12301), (16, 1500, 12288), (16, 64, 5200), (11, 4096, 6000), (13, 700, 2100), (16, 128, 16), (17, 200, 300), (33, 2048, 129),
         (64, 65, 1), (127, 255, 255), (129, 257, 511), (300, 1024, 3001), (333, 390, 2050), (700, 64, 1000), (1030, 65, 3001), (1153, 770, 2900),
         (1030, 130, 5003), (1281, 900, 4500), (2100, 70, 5000), (2100, 300, 5003), (2065, 1000, 4999), (1030, 192, 260), (300, 8320, 200)]


@pytest.mark.parametrize("m,d_in,d_out", SIZES)
def test_products(S, m, d_in, d_out):
    k = m + d_in + d_out
    X, W = _randn(k, m, d_in, dtype=TYPES[k % 3], scale=3), _randn(k + 1, d_out, d_in, dtype=TYPES[k // 3 % 3], scale=d_in ** -0.5)
    b, r = _randn(k + 2, d_out, dtype=TYPES[k // 9 % 3]), _randn(k + 3, m, d_out, dtype=TYPES[k // 2 % 3])
    w, p = S.prepare_int8(W), Q.product(X, W)
    for i, name in enumerate(Q.ACTS):
        _product(S, X, W, w, p, bias=b, activation=name, residual=r, out_dtype=TYPES[i % 3])
    _product(S, X, W, w, p, activation="silu", out_dtype=TYPES[(k + 1) % 3], rows=True)
    _product(S, X, W, w, p, residual=r, out_dtype=TYPES[(k + 2) % 3])
    _product(S, X, W, w, p, bias=b, out_dtype=TYPES[k % 3], rows=True)
    plain = S.int8_product(w, X, _ws(), out_dtype=TYPES[k % 3])
    assert torch.equal(S.int8_product(w, S.int8_rows(X), _ws(), out_dtype=TYPES[k % 3]), plain)


@pytest.mark.parametrize("m,d_in,d_out", [(m, i, -(-o // 2)) for m, i, o in SIZES] + [(1, 300, 4000), (9, 200, 160), (16, 200, 8000)])
def test_gated_products(S, m, d_in, d_out):
    k = m + d_in + d_out
    X = _randn(k, m, d_in, dtype=TYPES[k % 3], scale=3)
    Wg, Wu = (_randn(k + i, d_out, d_in, dtype=TYPES[k // 3 % 3], scale=d_in ** -0.5) for i in (1, 2))
    bg, bu = (_randn(k + i, d_out, dtype=TYPES[k // 9 % 3]) for i in (3, 4))
    r = _randn(k + 5, m, d_out, dtype=TYPES[k // 2 % 3])
    w, p = S.prepare_int8_gated(Wg, Wu), (Q.product(X, Wg), Q.product(X, Wu))
    for i, name in enumerate(Q.ACTS):
        _gated(S, X, Wg, Wu, w, p, gate_bias=bg, up_bias=bu, activation=name, out_dtype=TYPES[i % 3], rows=i % 2 == 1)
    _gated(S, X, Wg, Wu, w, p, out_dtype=TYPES[(k + 1) % 3])
    _gated(S, X, Wg, Wu, w, p, gate_bias=bg, residual=r, out_dtype=TYPES[(k + 2) % 3])
    _gated(S, X, Wg, Wu, w, p, up_bias=bu, rows=True)


@pytest.mark.parametrize("d_out,d_in", [(1, 1), (16, 64), (17, 65), (40, 128), (33, 4099), (257, 300)])
def test_prepared_gated_weights_bit_for_bit(S, d_out, d_in):
    for dtype in TYPES:
        Ws = [_randn(i, d_out, d_in, dtype=dtype) for i in (1, 2)]
        w = S.prepare_int8_gated(*Ws)
        torch.cuda.synchronize()
        rows = w.scale.numel()
        codes = R.weight_codes(w.codes.cpu().numpy(), rows, d_in)[0].reshape(-1, 2, 16, d_in)
        scale = w.scale.cpu().numpy().reshape(-1, 2, 16)
        for i, W in enumerate(Ws):
            c, s = R.rows_in_8_bits(R.as_f32(W))
            assert np.array_equal(codes[:, i].reshape(-1, d_in)[:d_out], c) and not codes[:, i].reshape(-1, d_in)[d_out:].any()
            assert np.array_equal(scale[:, i].reshape(-1)[:d_out], s) and not scale[:, i].reshape(-1)[d_out:].any()


@pytest.mark.parametrize("m,d_in,d_out", [(1, 300, 100), (7, 129, 65), (16, 64, 6001), (40, 250, 333), (200, 513, 2130), (1030, 130, 2700), (2100, 130, 2500)])
def test_strides_and_the_residual_in_place(S, m, d_in, d_out):
    """Rows apart and from an odd element on, the residual in the place of the outputs; nothing else is written."""
    for dtype in TYPES:
        X = _randn(1, m, d_in + 9, dtype=dtype)[:, 5:5 + d_in]
        Ws = [_randn(i, d_out, d_in + 4, dtype=dtype)[:, 1:1 + d_in] for i in (2, 3)]
        for gated in (False, True):
            whole = _randn(4, m + 2, d_out + 11, dtype=dtype)
            before, out = whole.clone(), whole[1:1 + m, 3:3 + d_out]
            r = before[1:1 + m, 3:3 + d_out]
            if gated:
                want = _gated(S, X, *Ws, residual=r, out_dtype=dtype)
                S.int8_gated_product(S.prepare_int8_gated(*Ws), X, _ws(), residual=out, out=out)
            else:
                want = _product(S, X, Ws[0], residual=r, activation="gelu", out_dtype=dtype)
                S.int8_product(S.prepare_int8(Ws[0]), X, _ws(), residual=out, activation="gelu", out=out)
            assert torch.equal(out, want)
            keep = torch.ones_like(whole, dtype=torch.bool)
            keep[1:1 + m, 3:3 + d_out] = False
            assert torch.equal(whole[keep], before[keep])


def test_rows_in_8_bits_bit_for_bit(S):
    for m, d in ((1, 1), (5, 129), (16, 64), (33, 4099), (3, 17000)):
        X = _randn(m, m, d, dtype=torch.bfloat16)
        rows = S.int8_rows(X)
        codes, scale = Q.coded(rows)
        want, wscale = R.rows_in_8_bits(R.as_f32(X))
        assert np.array_equal(codes, want) and np.array_equal(scale, wscale)
        Y = _randn(9, m, d, dtype=torch.bfloat16)
        assert S.int8_rows(Y, out=rows) is rows and np.array_equal(Q.coded(rows)[0], R.rows_in_8_bits(R.as_f32(Y))[0])


@pytest.mark.parametrize("m", [1, 3, 20, 150, 2100])
def test_rows_do_not_depend_on_each_other_and_bad_ones_are_flagged(S, m):
    from paper_2410_13056_amd import binding as B
    X, Ws = _randn(1, m, 300), [_randn(i, 2600, 300, dtype=torch.float16) for i in (2, 3)]
    w, g, status = S.prepare_int8(Ws[0]), S.prepare_int8_gated(*Ws), torch.zeros(1, dtype=torch.int32, device=DEV)
    calls = (lambda: S.int8_product(w, X, _ws(), activation="silu", status=status), lambda: S.int8_gated_product(g, X, _ws(), status=status))
    want = [c() for c in calls]
    assert status.item() == 0
    X[m - 1, 17], X[m - 1, 299] = float("nan"), float("-inf")
    for c, before in zip(calls, want):
        status.zero_()
        got = c()
        assert status.item() == B.STATUS_NONFINITE and torch.equal(got[:m - 1], before[:m - 1]) and got.isfinite().all()
    status.zero_()
    Ws[1][3, 5] = float("nan")
    S.prepare_int8_gated(*Ws, status)
    assert status.item() == B.STATUS_NONFINITE


def test_one_row_gives_what_it_gives_among_many(S):
    """The same row through every kernel: whatever the number of tokens, its outputs are the same bits."""
    X, Ws = _randn(1, 2100, 320, dtype=torch.float16), [_randn(i, 5000, 320, dtype=torch.float16) for i in (2, 3)]
    b, r = _randn(4, 5000), _randn(5, 2100, 5000)
    w, g = S.prepare_int8(Ws[0]), S.prepare_int8_gated(*Ws)
    for call in (lambda n: S.int8_product(w, X[:n], _ws(), bias=b, activation="gelu_tanh", residual=r[:n], out_dtype=torch.float32),
                 lambda n: S.int8_gated_product(g, X[:n], _ws(), gate_bias=b, residual=r[:n], out_dtype=torch.float32)):
        whole = call(2100)
        for n in (1, 2, 5, 16, 30, 64, 300, 700, 1100):
            assert torch.equal(call(n), whole[:n]), n


def test_outputs_beyond_32_bits_of_elements(S):
    m, d_out = 1 << 17, 16500
    X, Ws = torch.zeros((m, 64), dtype=torch.float16, device=DEV), [_randn(i, d_out, 64, dtype=torch.float16, scale=0.1) for i in (2, 3)]
    X[-3:] = _randn(1, 3, 64)
    out = torch.zeros((m, d_out), dtype=torch.float16, device=DEV)
    out[-3:] = 1
    S.int8_product(S.prepare_int8(Ws[0]), X, _ws(), residual=out, out=out, activation="gelu")
    want, bound = Q.finish(*Q.product(X[-3:], Ws[0]), None, "gelu", residual=np.ones((3, d_out)))
    Q.check(out[-3:], want, bound)
    assert not out[:-3].any()
    S.int8_gated_product(S.prepare_int8_gated(*Ws), X, _ws(), out=out)
    want, bound = Q.finish(*Q.product(X[-3:], Ws[0]), None, "silu", *Q.product(X[-3:], Ws[1]))
    Q.check(out[-3:], want, bound)
    assert not out[:-3].any()


def test_zero_rows_and_weights(S):
    for m in (1, 40, 300):
        X, Ws = _randn(1, m, 200), [_randn(i, 50, 200) for i in (2, 3)]
        X[m // 2] = 0
        Ws[0][7] = 0
        b = _randn(4, 50)
        got = _product(S, X, Ws[0], bias=b, out_dtype=torch.float32)
        assert torch.equal(got[m // 2], b) and torch.equal(got[:, 7], b[7].expand(m))
        assert not _gated(S, X, *Ws, out_dtype=torch.float32)[:, 7].any()


def test_no_rows(S):
    Ws = [_randn(i, 40, 64) for i in (1, 2)]
    X = torch.empty((0, 64), device=DEV)
    for x in (X, S.int8_rows(X)):
        assert S.int8_product(S.prepare_int8(Ws[0]), x, _ws(), activation="silu").shape == (0, 40)
        assert S.int8_gated_product(S.prepare_int8_gated(*Ws), x, _ws()).shape == (0, 40)


@pytest.mark.parametrize("m", [1, 6, 30, 70, 260, 2100])
def test_another_stream_and_graph_replays(S, m):
    """Two graphs that share a workspace, replayed one after the other, several times, with eager work between."""
    X, Ws = _randn(1, m, 500, dtype=torch.float16), [_randn(i, 2600, 500, dtype=torch.float16) for i in (2, 3)]
    w, g, ws, r = S.prepare_int8(Ws[0]), S.prepare_int8_gated(*Ws), _ws(), _randn(4, m, 2600)
    calls = (lambda ws, out=None: S.int8_product(w, X, ws, activation="silu", residual=r, out=out),
             lambda ws, out=None: S.int8_gated_product(g, X, ws, out=out))
    want = [c(ws) for c in calls]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [c(_ws()) for c in calls]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    outs, graphs = [torch.empty_like(t) for t in want], []
    for c, out in zip(calls, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c(ws, out)
        graphs.append(graph)
    for k in range(3):
        for t in outs:
            t.zero_()
        X.copy_(_randn(10 + k, m, 500, dtype=torch.float16))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out, c(_ws())) for c, out in zip(calls, outs))
