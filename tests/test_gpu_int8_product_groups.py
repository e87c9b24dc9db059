"""Sizes that launch the products in which groups of wavefronts share the depth - tiles of 64 x 64 to 128 x 128 in two and three
groups, two pieces by two - with depths that leave a group little or nothing, plain, with an epilogue and gated; and tokens that are coded within the one launch.  Exact sums:
the plain outputs are bit for bit those of the codes."""
import pytest
import torch

import test_gpu_int8_finish as T
import test_gpu_int8_product as P
from test_gpu_int8_finish import S  # noqa: F401

pytestmark = pytest.mark.gpu

DEV = "cuda"
SIZES = [(700, d, 1000) for d in (1, 128, 129, 256, 300, 1000)] + [(100, 5120, 5120), (160, 130, 5333)] + \
        [(333, d, 3001) for d in (64, 256, 390, 1025)] + [(290, 700, 4099)] + \
        [(150, d, 11008) for d in (100, 200, 1030)] + \
        [(64, 8192, 1024), (40, 6200, 300), (17, 7000, 130), (64, 300, 1024), (250, 1, 900), (40, 300, 8192), (24, 6150, 5000)] + \
        [(1, 6144, 40), (1, 6145, 40), (1, 16000, 300), (1, 20000, 33), (1, 32768, 17), (1, 32769, 17), (2, 20000, 4000), (2, 32768, 30),
         (2, 30000, 4200), (16, 700, 5130), (13, 1000, 8192), (16, 200, 8200)]


ROUNDS = [(m, d, n) for m, n in [(330, 3000), (50, 16500), (145, 11001), (700, 4000), (690, 4003)] for d in (1, 129, 300, 515, 1100)] + \
         [(333, 4099, 3001), (96, 2000, 8200), (64, 1000, 28600), (400, 1000, 5003)]


@pytest.mark.parametrize("m,d_in,d_out", SIZES + ROUNDS)
def test_products(S, m, d_in, d_out):  # noqa: F811
    k = m + d_in + d_out
    X = T._randn(k, m, d_in, dtype=T.TYPES[k % 3], scale=3)
    Ws = [T._randn(k + i, d_out, d_in, dtype=T.TYPES[k // 3 % 3], scale=d_in ** -0.5) for i in (1, 2)]
    b, r, out = T._randn(k + 3, d_out), T._randn(k + 4, m, d_out), T.TYPES[k // 2 % 3]
    w = S.prepare_int8(Ws[0])
    P._check(S, X, Ws[0], torch.float32, w)
    T._product(S, X, Ws[0], w, bias=b, activation="gelu_tanh", residual=r, out_dtype=out)
    T._gated(S, X, *Ws, residual=r, out_dtype=out)
    if d_out > 1000:
        half = [W[:(d_out + 1) // 2] for W in Ws]
        T._gated(S, X, *half, gate_bias=b[:(d_out + 1) // 2], out_dtype=torch.float32)


def test_one_row_in_every_tile(S):  # noqa: F811
    """As below, by the tiles that take a round of the units."""
    X, W = T._randn(1, 1000, 1000, dtype=torch.float16), T._randn(2, 11008, 1000, dtype=torch.float16)
    w = S.prepare_int8(W)
    whole = S.int8_product(w, X, T._ws(), out_dtype=torch.float32)
    for n in (40, 64, 96, 144, 150, 200, 256):
        assert torch.equal(S.int8_product(w, X[:n], T._ws(), out_dtype=torch.float32), whole[:n]), n


def test_groups_add_up_to_the_same_sums(S):  # noqa: F811
    """A row's outputs do not depend on which kernel the number of rows asks for."""
    X, W = T._randn(1, 700, 1000, dtype=torch.float16), T._randn(2, 3001, 1000, dtype=torch.float16)
    w = S.prepare_int8(W)
    whole = S.int8_product(w, X, T._ws(), out_dtype=torch.float32)
    for n in (1, 2, 10, 30, 64, 200, 300, 333, 500):
        assert torch.equal(S.int8_product(w, X[:n], T._ws(), out_dtype=torch.float32), whole[:n]), n


@pytest.mark.parametrize("out", T.TYPES)
@pytest.mark.parametrize("m,d_out", [(700, 3000), (330, 3001), (2100, 4100), (100, 300)])
def test_outputs_at_any_address(S, m, d_out, out):  # noqa: F811
    """Outputs that cannot be written four at once are the bits of those that can, and nothing beside them is written.  (Those of
    FP16 are not the ones in 32 bits rounded: their last multiplication and its rounding to FP16 are one.)"""
    X, W = T._randn(m, m, 300, dtype=torch.float16), T._randn(d_out, d_out, 300, dtype=torch.float16)
    w = S.prepare_int8(W)
    want = torch.empty((m, (d_out + 3) // 4 * 4), dtype=out, device=DEV)[:, :d_out]
    S.int8_product(w, X, T._ws(), out=want)
    exact = S.int8_product(w, X, T._ws(), out_dtype=torch.float32)
    assert ((want.double() - exact.double()).abs() <= exact.abs().double() * torch.finfo(out).eps / 2 * (1 + 2.0 ** -9) + 2.0 ** -24).all()
    for columns, first in [(d_out + 1, 0), (d_out + 1, 1), (d_out + 6, 3), (d_out + 8 - d_out % 4, 4)]:
        room = torch.full((m, columns), -7.0, dtype=out, device=DEV)
        place = room[:, first:first + d_out]
        S.int8_product(w, X, T._ws(), out=place)
        assert torch.equal(place, want)
        place.fill_(-7.0)
        assert torch.equal(room, torch.full_like(room, -7.0))


@pytest.mark.parametrize("kind", T.TYPES)
@pytest.mark.parametrize("m,d", [(2048, 4096), (2051, 130), (2050, 4097), (2100, 8190), (2065, 16384), (2049, 9001), (2047, 700), (300, 16385), (2048, 20000)])
def test_many_rows_are_coded_as_few(S, m, d, kind):  # noqa: F811
    """Codes, scales and flags of a row do not depend on the number of rows, and a row that is not finite is none of its neighbours' matter."""
    X = T._randn(m + d, m, d, dtype=kind, scale=5)
    X[5, d // 2], X[6, 0], X[m - 1, d - 1], X[9] = float("inf"), float("nan"), -float("inf"), 0
    X = torch.cat([X, X], 1)[:, 1:d + 1] if d % 2 else X
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    rows = S.int8_rows(X, status=status)
    pieces = rows.codes.view(-1, rows.codes.numel() // ((m + 15) // 16))
    assert status.item()
    for i in [0, 16 * (m // 32), (m - 1) // 16 * 16]:
        some = S.int8_rows(X[i:i + 16])
        assert torch.equal(some.codes, pieces[i // 16]) and torch.equal(some.scale, rows.scale[i:i + 16])
    status.zero_()
    S.int8_rows(X[16:m - 16], status=status)
    assert not status.item()
