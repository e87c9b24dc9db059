"""Products in 8-bit integers through the public calls: codes bit for bit, outputs against the same sums in 64 bits."""
import numpy as np
import pytest
import torch

import serving_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
# (float)sum * sx * sw: one rounding of the sum and two of the products, then the output's own
ROUND = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
FEW = 4 * 2.0 ** -24
TINIEST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _check(S, X, W, out_dtype, w=None, ws=None, **kw):
    from paper_2410_13056_amd import binding as B
    w = w or S.prepare_int8(W)
    Y = S.int8_product(w, X, ws or B.Workspace(DEV), out_dtype=out_dtype, **kw)
    torch.cuda.synchronize()
    cx, sx = R.rows_in_8_bits(R.as_f32(X))
    cw, sw = R.rows_in_8_bits(R.as_f32(W))
    want = (cx.astype(np.float64) @ cw.T.astype(np.float64)) * sx[:, None].astype(np.float64) * sw
    got = Y.double().cpu().numpy()
    off = np.abs(got - want)
    assert Y.dtype == out_dtype and (off <= np.abs(want) * (ROUND[out_dtype] + FEW) + TINIEST[out_dtype]).all(), off.max()
    return Y


SIZES = [(1, 1, 1), (1, 64, 16), (1, 127, 70), (1, 4096, 1000), (2, 63, 17), (3, 1030, 515), (5, 129, 33), (8, 512, 64), (13, 700, 2100),
         (16, 128, 16), (17, 200, 300), (31, 96, 250), (33, 2048, 129), (64, 65, 1), (65, 4099, 130), (100, 1, 257),
         (127, 255, 255), (128, 256, 256), (129, 257, 511), (257, 640, 384), (300, 1024, 3001), (513, 320, 770), (1030, 192, 260)]
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.mark.parametrize("m,d_in,d_out", SIZES)
def test_sizes(S, m, d_in, d_out):
    g = _gen(m * 7 + d_in)
    kind = (m + d_in + d_out) % 9
    X = (torch.randn((m, d_in), generator=g, device=DEV) * 3).to(TYPES[kind % 3])
    W = (torch.randn((d_out, d_in), generator=g, device=DEV) * 0.02).to(TYPES[kind // 3])
    for out in TYPES:
        _check(S, X, W, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d_out,d_in", [(1, 1), (16, 64), (17, 65), (40, 128), (33, 4099), (257, 300)])
def test_prepared_weight_bit_for_bit(S, d_out, d_in, dtype):
    W = (torch.randn((d_out, d_in), generator=_gen(d_in), device=DEV) * 0.05).to(dtype)
    w = S.prepare_int8(W)
    torch.cuda.synchronize()
    codes, scale = R.rows_in_8_bits(R.as_f32(W))
    got, below, beyond = R.weight_codes(w.codes.cpu().numpy(), d_out, d_in)
    assert np.array_equal(got, codes) and not below.any() and not beyond.any()
    assert np.array_equal(w.scale.cpu().numpy(), scale)


def test_strides_of_inputs_and_outputs(S):
    g = _gen(3)
    for m, d_in, d_out, off in ((1, 300, 100, 1), (7, 129, 65, 3), (40, 250, 333, 5), (200, 513, 130, 7), (600, 130, 270, 2)):
        X = torch.randn((m, d_in + 9), generator=g, device=DEV).half()[:, off:off + d_in]
        W = torch.randn((d_out, d_in + 4), generator=g, device=DEV).half()[:, 1:1 + d_in]
        whole = torch.full((m + 2, d_out + 11), 7.0, device=DEV, dtype=torch.bfloat16)
        out = whole[1:1 + m, off:off + d_out]
        _check(S, X, W, torch.bfloat16, out=out)
        keep = torch.ones_like(whole, dtype=torch.bool)
        keep[1:1 + m, off:off + d_out] = False
        assert (whole[keep] == 7.0).all()                       # nothing else was written


def test_largest_sums_are_exact(S):
    d_in = 131072
    X, W = torch.full((2, d_in), 2.0, device=DEV), torch.full((20, d_in), -0.5, device=DEV)
    Y = _check(S, X, W, torch.float32)
    assert (Y == np.float32(-127 * 127 * d_in) * np.float32(2 / np.float32(127)) * np.float32(0.5 / np.float32(127))).all()


def test_zero_tiny_and_large_rows(S):
    g = _gen(5)
    for m in (1, 5, 40, 300):
        X = torch.randn((m, 200), generator=g, device=DEV)
        X[m // 2] = 0
        X[0] *= 1e-30
        X[m - 1] *= 1e37
        W = torch.randn((50, 200), generator=g, device=DEV) * 1e-3
        W[7] = 0
        Y = _check(S, X, W, torch.float32)
        assert (Y[:, 7] == 0).all()


@pytest.mark.parametrize("m", [1, 3, 20, 150])
def test_non_finite_inputs_are_flagged_and_stay_in_their_rows(S, m):
    from paper_2410_13056_amd import binding as B
    g = _gen(11)
    X, W = torch.randn((m, 300), generator=g, device=DEV), torch.randn((70, 300), generator=g, device=DEV).half()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    _check(S, X, W, torch.float32, status=status)
    assert status.item() == 0
    X[m - 1, 17], X[m - 1, 200], X[m - 1, 299] = float("nan"), float("inf"), float("-inf")
    _check(S, X, W, torch.float32, status=status)               # NaN codes 0, infinities +-127 of the finite scale
    assert status.item() == B.STATUS_NONFINITE
    status.zero_()
    W[3, 5] = float("nan")
    w = S.prepare_int8(W, status)
    torch.cuda.synchronize()
    assert status.item() == B.STATUS_NONFINITE
    codes, _ = R.rows_in_8_bits(R.as_f32(W))
    assert np.array_equal(R.weight_codes(w.codes.cpu().numpy(), 70, 300)[0], codes)


def test_another_stream_and_graph_replays(S):
    from paper_2410_13056_amd import binding as B
    g = _gen(13)
    for m in (1, 6, 70, 260):
        X, W = torch.randn((m, 500), generator=g, device=DEV).half(), torch.randn((260, 500), generator=g, device=DEV).half()
        w, ws = S.prepare_int8(W), B.Workspace(DEV)
        want = S.int8_product(w, X, ws).clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = S.int8_product(w, X, B.Workspace(DEV))
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        out, graph = torch.empty_like(want), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            S.int8_product(w, X, ws, out=out)
        for k in range(3):
            out.zero_()
            X.copy_(torch.randn((m, 500), generator=g, device=DEV).half())
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, S.int8_product(w, X, B.Workspace(DEV)))


def test_refusals(S):
    from paper_2410_13056_amd import binding as B
    w, ws = S.prepare_int8(torch.randn((40, 64), device=DEV)), B.Workspace(DEV)
    with pytest.raises(ValueError):
        S.int8_product(w, torch.randn((2, 63), device=DEV), ws, out=torch.empty((2, 40), device=DEV)[:, :39])
    with pytest.raises(ValueError):
        S.int8_product(w, torch.randn((2, 64), device=DEV), ws, out=torch.empty((3, 40), device=DEV))
    with pytest.raises(TypeError):
        S.int8_product(w, torch.zeros((2, 64), device=DEV, dtype=torch.int32), ws)
    with pytest.raises(ValueError):
        S.int8_product(w, torch.randn((64, 2), device=DEV).t(), ws)
    with pytest.raises(ValueError):
        S.int8_product(w, torch.randn((2, 64)), ws, out=torch.empty((2, 40), device=DEV))
    assert S.int8_product(w, torch.empty((0, 64), device=DEV), ws).shape == (0, 40)
