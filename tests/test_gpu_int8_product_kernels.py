"""Sizes that between them launch every kernel of the product in 8-bit integers, with edges that are part full.  The
rule: up to 2 tokens and 16384 inputs one launch; up to 16 tokens 2 or 1 pieces of 16 outputs by 8 or 16 wavefronts, from 768
and 320 pieces on; up to 32 tokens 4 x 2 pieces; beyond, the largest of 256 x 256, 256 x 128, 128 x 128 and 64 x 64 whose tiles fill
256 compute units, 4 x 2 pieces else."""
import pytest
import torch

import test_gpu_int8_product as T

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


SIZES = [(2100, 70, 5000), (2100, 300, 5003), (2304, 128, 5120), (2065, 1000, 4999),      # 256 x 256: 1, 3, 1 and 8 pairs of steps
         (1030, 130, 5003), (1100, 64, 5120), (1281, 900, 4500),                          # 256 x 128
         (1030, 65, 3001), (1024, 128, 3136), (1153, 770, 2900),                     # 128 x 128
         (700, 64, 1000), (333, 390, 2050),                                               # 64 x 64
         (5, 129, 12301), (16, 1500, 12288), (9, 64, 14000),                              # 2 pieces, 8 wavefronts
         (16, 64, 5200), (3, 1100, 5121), (11, 4096, 6000),                               # 1 piece, 8 wavefronts
         (3, 9000, 40), (40, 16384, 33), (17, 12300, 130), (300, 8320, 200),              # codes of 4 times 4096 inputs a row
         (5, 20000, 48), (2, 16384, 50), (1, 16385, 40), (2, 16400, 64), (70, 16500, 100)]  # and of longer rows


@pytest.mark.parametrize("m,d_in,d_out", SIZES)
def test_sizes_of_every_kernel(S, m, d_in, d_out):
    g = T._gen(m + d_in)
    kind = (m + d_in + d_out) % 9
    X = (torch.randn((m, d_in), generator=g, device=DEV) * 3).to(T.TYPES[kind % 3])
    W = (torch.randn((d_out, d_in), generator=g, device=DEV) * 0.02).to(T.TYPES[kind // 3])
    w = S.prepare_int8(W)
    for out in T.TYPES:
        T._check(S, X, W, out, w)
    gap = torch.full((m, d_out + 3), 7.0, device=DEV)                    # rows of odd stride, from an odd element on
    T._check(S, X, W, torch.float32, w, out=gap[:, 1:1 + d_out])
    assert (gap[:, 0] == 7).all() and (gap[:, 1 + d_out:] == 7).all()


@pytest.mark.parametrize("m,d_in,d_out", [(2100, 300, 5003), (1030, 130, 5003), (1030, 65, 3001), (5, 129, 12301), (16, 64, 5200), (40, 9000, 100)])
def test_graph_replays_of_every_kernel(S, m, d_in, d_out):
    from paper_2410_13056_amd import binding as B
    g = T._gen(17)
    X, W = torch.randn((m, d_in), generator=g, device=DEV).half(), torch.randn((d_out, d_in), generator=g, device=DEV).half()
    w, ws = S.prepare_int8(W), B.Workspace(DEV)
    out = S.int8_product(w, X, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.int8_product(w, X, ws, out=out)
    for k in range(3):
        out.zero_()
        X.copy_(torch.randn((m, d_in), generator=g, device=DEV).half())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, S.int8_product(w, X, B.Workspace(DEV)))


def test_the_call_without_a_prepared_layer(S):
    from paper_2410_13056_amd import binding as B
    X, W = torch.randn((7, 100), device=DEV).half(), torch.randn((33, 100), device=DEV).half()
    w, Y = S.prepare_int8(W), torch.empty((7, 33), device=DEV)
    B.int8_product(X, w.codes, w.scale, Y, B.Workspace(DEV))
    assert torch.equal(Y, S.int8_product(w, X, out_dtype=torch.float32))
    with pytest.raises(ValueError):
        B.int8_product(X, w.codes[:-1], w.scale, Y, B.Workspace(DEV))
