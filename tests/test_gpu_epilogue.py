"""The epilogue by itself, through the public call, against 64 bits."""
import itertools

import pytest
import torch

import feed_forward_reference as Q

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


def _check(S, Y, bias=None, name=None, times=None, times_bias=None, residual=None, out_dtype=None, out=None):
    want, bound = Q.finish(Q.f64(Y), 0.0, Q.f64(bias), name, Q.f64(times), 0.0, Q.f64(times_bias), Q.f64(residual))
    got = S.epilogue(Y, bias, name, times, times_bias, residual, out_dtype, out)
    torch.cuda.synchronize()
    Q.check(got, want, bound)
    return got


@pytest.mark.parametrize("m,d", [(1, 1), (1, 7), (2, 8), (3, 9), (1, 13824), (17, 130), (64, 4099), (300, 1000), (1, 65537), (70000, 3), (2100, 2053)])
def test_sizes(S, m, d):
    k = m + d
    for name in Q.ACTS:
        _check(S, _randn(k, m, d, scale=3), name=name)
        _check(S, _randn(k, m, d, scale=3, dtype=TYPES[k % 3]), _randn(1, d, dtype=TYPES[k // 3 % 3]), name, _randn(2, m, d, dtype=TYPES[(k + 1) % 3]),
               _randn(3, d, dtype=TYPES[(k + 2) % 3]), _randn(4, m, d, dtype=TYPES[k // 2 % 3]), TYPES[k // 5 % 3])


@pytest.mark.parametrize("y,t,r,out", list(itertools.product(TYPES, TYPES, TYPES, TYPES)))
def test_types(S, y, t, r, out):
    m, d = 5, 77
    _check(S, _randn(1, m, d, dtype=y), _randn(2, d, dtype=t), "silu", _randn(3, m, d, dtype=t), _randn(4, d, dtype=r), _randn(5, m, d, dtype=r), out)


@pytest.mark.parametrize("name", Q.ACTS)
def test_activations_over_the_whole_range(S, name):
    """From the smallest magnitudes to the largest, both signs, as the definition has them within fp32's bounds."""
    mags = torch.cat([torch.logspace(-44, 38, 4000, dtype=torch.float64), torch.linspace(0, 120, 6000, dtype=torch.float64)]).float()
    v = torch.cat([mags, -mags]).view(2, -1).to(DEV)
    got = _check(S, v, name=name)
    assert got.isfinite().all()


@pytest.mark.parametrize("name", Q.ACTS)
def test_values_that_are_no_numbers(S, name):
    """NaN stays NaN; plus infinity is itself; minus infinity 0 or itself without the limit that the header leaves out."""
    Y = _randn(1, 4, 40)
    Y[0, 3], Y[1, 8], Y[2, 9] = float("nan"), float("inf"), float("-inf")
    got = S.epilogue(Y, activation=name)
    assert got[0, 3].isnan() and got[1, 8] == float("inf")
    low = got[2, 9].item()
    assert low == {None: float("-inf"), "relu": 0.0}.get(name) if name in (None, "relu") else got[2, 9].isnan()
    Y[0, 3], Y[1, 8], Y[2, 9] = 0.0, 0.0, 0.0
    fine = torch.ones_like(Y, dtype=torch.bool)
    fine[0, 3] = fine[1, 8] = fine[2, 9] = False
    assert torch.equal(got[fine], S.epilogue(Y, activation=name)[fine])


def test_strides_and_places(S):
    for m, d, dtype in ((5, 100, torch.float32), (7, 4001, torch.float16), (300, 40, torch.bfloat16)):
        whole = {n: _randn(i, m + 2, d + 9, dtype=dtype) for i, n in enumerate(("Y", "times", "residual", "out"))}
        view = {n: t[1:1 + m, 3:3 + d] for n, t in whole.items()}
        before = whole["out"].clone()
        want = _check(S, view["Y"], name="gelu", times=view["times"], residual=view["residual"], out=view["out"]).clone()
        keep = torch.ones_like(before, dtype=torch.bool)
        keep[1:1 + m, 3:3 + d] = False
        assert torch.equal(whole["out"][keep], before[keep])
        for place in ("Y", "times", "residual"):
            t = {n: v.clone()[1:1 + m, 3:3 + d] for n, v in whole.items()}
            got = S.epilogue(t["Y"], None, "gelu", t["times"], None, t["residual"], out=t[place])
            assert got is t[place] and torch.equal(got, want)


def test_rows_beyond_32_bits_of_elements(S):
    m, d = 75000, 28700
    Y, U = torch.zeros((m, d), dtype=torch.float16, device=DEV), torch.ones((m, d), dtype=torch.float16, device=DEV)
    Y[-2:], U[-2:] = _randn(1, 2, d), _randn(2, 2, d)
    got = S.epilogue(Y, activation="silu", times=U)
    want, bound = Q.finish(Q.f64(Y[-2:]), 0.0, None, "silu", Q.f64(U[-2:]))
    Q.check(got[-2:], want, bound)
    assert not got[:-2].any()


def test_no_rows_and_no_columns(S):
    for m, d in ((0, 8), (8, 0), (0, 0)):
        assert S.epilogue(torch.empty((m, d), device=DEV), activation="silu").shape == (m, d)


def test_another_stream_and_graph_replays(S):
    Y, U = _randn(1, 30, 500), _randn(2, 30, 500)
    want = S.epilogue(Y, activation="silu", times=U)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = S.epilogue(Y, activation="silu", times=U)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out, graph = torch.empty_like(Y), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.epilogue(Y, activation="silu", times=U, out=out)
    for k in range(3):
        out.zero_()
        Y.copy_(_randn(10 + k, 30, 500))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, S.epilogue(Y, activation="silu", times=U))
