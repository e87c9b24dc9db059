"""Sizes on both sides of the lines that the choice of kernels is made by: one token by 8 or 16 wavefronts; tiles of 64 x 64 by one or two
groups of wavefronts; tiles of 128 x 128 of one group, up to two a unit and more."""
import pytest
import torch

import test_gpu_int8_finish as T
import test_gpu_int8_product as P
from test_gpu_int8_finish import S  # noqa: F401

pytestmark = pytest.mark.gpu

ONE = [(1, d, n) for d in (1024, 1025, 2048, 2049, 4096, 4097, 6144) for n in (4096, 4097, 8200)] + [(1, 6145, 4100), (1, 70, 5000)]
TILES = [(128, 130, 4700), (128, 4200, 5000), (129, 4030, 3401), (129, 4032, 3400), (333, 4096, 2050), (200, 4200, 3300), (140, 6000, 4000),
         (100, 1, 5000), (600, 3000, 1000), (600, 5000, 999)] + \
        [(700, 200, 11100), (600, 1000, 6500), (700, 1100, 11000), (1500, 300, 11008)]


@pytest.mark.parametrize("m,d_in,d_out", ONE + TILES)
def test_products(S, m, d_in, d_out):  # noqa: F811
    k = m + d_in + d_out
    X = T._randn(k, m, d_in, dtype=T.TYPES[k % 3], scale=3)
    Ws = [T._randn(k + i, d_out, d_in, dtype=T.TYPES[k // 3 % 3], scale=d_in ** -0.5) for i in (1, 2)]
    b, r, out = T._randn(k + 3, d_out), T._randn(k + 4, m, d_out), T.TYPES[k // 2 % 3]
    w = S.prepare_int8(Ws[0])
    P._check(S, X, Ws[0], torch.float32, w)
    T._product(S, X, Ws[0], w, bias=b, activation="silu", residual=r, out_dtype=out)
    half = [W[:(d_out + 1) // 2] for W in Ws]
    T._gated(S, X, *half, gate_bias=b[:(d_out + 1) // 2], out_dtype=out)


def test_a_graph_of_each(S):  # noqa: F811
    for m, d_in, d_out in ((1, 4096, 4096), (1, 5120, 8200), (128, 300, 4700), (333, 4096, 2050), (700, 200, 11100)):
        X, W = T._randn(1, m, d_in, dtype=torch.float16), T._randn(2, d_out, d_in, dtype=torch.float16)
        w, ws = S.prepare_int8(W), T._ws()
        out = S.int8_product(w, X, ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            S.int8_product(w, X, ws, out=out)
        for k in range(3):
            out.zero_()
            X.copy_(T._randn(10 + k, m, d_in))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, S.int8_product(w, X, T._ws()))
