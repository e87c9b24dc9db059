"""The root-mean-square norm through the public call: bit for bit, since its one sum is in 64 bits and every other step rounds
to fp32 where the definition says so."""
import numpy as np
import pytest
import torch

import feed_forward_reference as Q
import serving_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float16, torch.bfloat16, torch.float32]
EPS = 1e-5


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _randn(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def _same(got, want, dtype=None):
    """Equal, NaN where NaN is expected."""
    w = torch.from_numpy(want) if isinstance(want, np.ndarray) else want
    w = w.to(dtype or got.dtype)
    assert torch.equal(got.cpu().nan_to_num(nan=77.0), w.nan_to_num(nan=77.0)) and torch.equal(got.cpu().isnan(), w.isnan())


def _check(S, X, weight=None, add=None, sum_dtype=None, out_dtype=None, eps=EPS, status=None):
    """Values and rows in 8 bits."""
    kw = dict(add=add, status=status)
    if sum_dtype is not None:
        kw["sum_out"] = torch.empty(X.shape, dtype=sum_dtype, device=DEV)
    got = S.rms_norm(X, weight, eps, out_dtype=out_dtype, **kw)
    rows = S.rms_norm(X, weight, eps, coded=True, **kw)
    if add is not None:
        sum_dtype = sum_dtype or X.dtype
        (got, total), (rows, again) = got, rows
        assert total.dtype == sum_dtype and torch.equal(total.nan_to_num(nan=77.0), again.nan_to_num(nan=77.0))
    y, s = Q.norm(X, add, weight, eps, sum_dtype)
    if add is not None:
        _same(total, s)
    assert got.dtype == (out_dtype or X.dtype)
    _same(got, y)
    codes, scale = Q.coded(rows)
    want, wscale = R.rows_in_8_bits(y)
    assert np.array_equal(scale, wscale) and np.array_equal(codes, want)
    return got


SIZES = [(1, 1), (1, 7), (2, 64), (1, 2048), (3, 2049), (17, 129), (16, 4096), (5, 4097), (33, 5120), (1, 8192), (4, 8191), (31, 8200),
         (2, 16384), (3, 16385), (1, 28672), (2, 32768), (3, 32769), (2, 40003), (1, 131072), (700, 300), (4099, 64), (1, 2047)]


@pytest.mark.parametrize("m,d", SIZES)
def test_sizes(S, m, d):
    k = m + d
    X, A = _randn(k, m, d, dtype=TYPES[k % 3]), _randn(k + 1, m, d, dtype=TYPES[k // 3 % 3])
    W = _randn(k + 2, d, dtype=TYPES[k // 9 % 3])
    _check(S, X)
    _check(S, X, W, A, out_dtype=TYPES[(k + 1) % 3])
    _check(S, X, W, None, None, TYPES[(k + 2) % 3])


@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("a", TYPES)
@pytest.mark.parametrize("out", TYPES)
def test_types(S, x, a, out):
    X, A, W = _randn(1, 21, 770, dtype=x), _randn(2, 21, 770, dtype=a), _randn(3, 770, dtype=a)
    for s in TYPES:
        _check(S, X, W, A, s, out)


@pytest.mark.parametrize("d", [100, 1001, 9000, 33001])
def test_strides_and_places(S, d):
    """Rows apart and from an odd element on; the sum or the norm in the place of either input; nothing else is written."""
    m = 9
    for dtype in TYPES:
        whole = {n: _randn(i + d, m + 2, d + 11, dtype=dtype) for i, n in enumerate("XAYS")}
        view = {n: t[1:1 + m, 3:3 + d] for n, t in whole.items()}
        before = {n: t.clone() for n, t in whole.items()}
        W = _randn(5, d, dtype=dtype)
        y, s = Q.norm(view["X"], view["A"], W, EPS, dtype)
        S.rms_norm(view["X"], W, EPS, add=view["A"], out=view["Y"], sum_out=view["S"])
        _same(view["Y"], y)
        _same(view["S"], s)
        keep = torch.ones_like(whole["X"], dtype=torch.bool)
        keep[1:1 + m, 3:3 + d] = False
        for n in "XAYS":
            assert torch.equal(whole[n][keep], before[n][keep])
        for place in "XA":
            for other in "XA":
                t = {n: before[n].clone()[1:1 + m, 3:3 + d] for n in "XA"}
                if place != other:
                    S.rms_norm(t["X"], W, EPS, add=t["A"], out=t[other], sum_out=t[place])
                    _same(t[other], y)
                else:
                    S.rms_norm(t["X"], W, EPS, add=t["A"], sum_out=t[place])
                _same(t[place], s)
            t = {n: before[n].clone()[1:1 + m, 3:3 + d] for n in "XA"}
            rows, total = S.rms_norm(t["X"], W, EPS, add=t["A"], coded=True, sum_out=t[place])
            assert total is t[place] and np.array_equal(Q.coded(rows)[0], R.rows_in_8_bits(y)[0])
            _same(total, s)


def test_zero_tiny_and_large_rows(S):
    for d in (64, 5000, 40000):
        X = _randn(d, 6, d)
        X[1] = 0
        X[2] *= 1e-30
        X[3] *= 1e37
        X[4, 0] = 3e38
        _check(S, X, _randn(3, d))
        _check(S, X, _randn(3, d), eps=2.0 ** -126)
        _check(S, X[:2], torch.full((d,), 3e38, device=DEV))        # products beyond fp32: infinities, codes +-127


@pytest.mark.parametrize("m,d", [(1, 64), (40, 3000), (3, 40001)])
def test_non_finite_rows_are_flagged_and_stay_in_their_rows(S, m, d):
    from paper_2410_13056_amd import binding as B
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    X = _randn(m, m, d)
    _check(S, X, status=status)
    assert status.item() == 0
    X[m - 1, d - 1] = float("inf")
    X[0, 5] = float("nan") if m > 1 else X[0, 5]
    for coded in (False, True):
        status.zero_()
        S.rms_norm(X, None, EPS, coded=coded, status=status)
        assert status.item() == B.STATUS_NONFINITE
    _check(S, X, _randn(2, d), status=status)
    W = _randn(2, d)
    W[3] = float("nan")
    status.zero_()
    _check(S, X[1:2], W, status=status)
    assert m == 1 or status.item() == B.STATUS_NONFINITE


def test_no_rows(S):
    X = torch.empty((0, 64), device=DEV)
    Y, total = S.rms_norm(X, add=X)
    assert Y.shape == total.shape == (0, 64)
    assert S.rms_norm(X, coded=True).rows == 0


def test_rows_beyond_32_bits_of_elements(S):
    m, d = 262400, 8200                                              # 2.15e9 elements
    X = torch.zeros((m, d), dtype=torch.float16, device=DEV)
    X[-3:] = _randn(1, 3, d, dtype=torch.float16)
    Y = S.rms_norm(X, _randn(2, d))
    rows = S.rms_norm(X, _randn(2, d), coded=True)
    y, _ = Q.norm(X[-3:], None, _randn(2, d), 1e-6, None)
    _same(Y[-3:], y)
    assert not Y[:-3].any()
    last = rows.codes.view(-1, 16 * ((d + 127) // 128 * 128))[-1].cpu().numpy()
    codes, _, _ = R.weight_codes(last, 16, d)
    assert np.array_equal(codes[-3:], R.rows_in_8_bits(y)[0])


def test_another_stream_and_graph_replays(S):
    for m, d in ((1, 500), (40, 9000), (3, 33000)):
        X, A, W = _randn(1, m, d, dtype=torch.float16), _randn(2, m, d, dtype=torch.float16), _randn(3, d)
        want, total = S.rms_norm(X, W, EPS, add=A)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got, t2 = S.rms_norm(X, W, EPS, add=A)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(total, t2)
        out, sum_out, rows = torch.empty_like(want), torch.empty_like(want), S.rms_norm(X, W, EPS, coded=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            S.rms_norm(X, W, EPS, add=A, out=out, sum_out=sum_out)
            S.rms_norm(X, W, EPS, coded=True, out=rows)
        for k in range(3):
            out.zero_()
            rows.codes.zero_()
            X.copy_(_randn(10 + k, m, d, dtype=torch.float16))
            graph.replay()
            torch.cuda.synchronize()
            want, total = S.rms_norm(X, W, EPS, add=A)
            assert torch.equal(out, want) and torch.equal(sum_out, total)
            assert torch.equal(rows.codes, S.rms_norm(X, W, EPS, coded=True).codes)
