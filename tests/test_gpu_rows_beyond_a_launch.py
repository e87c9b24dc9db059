"""As many rows as the limits allow, which are more than one launch has lanes for: the whole is what its parts are."""
import pytest
import torch

from test_gpu_rms_norm import DEV, S, _randn  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = (1 << 24) - 1
PART = 1 << 20


def _same_codes(whole, part, at):
    """`part` holds the rows of `whole` from `at` on (a multiple of 16)."""
    per = part.codes.numel() // -(-part.rows // 16)                         # bytes of 16 rows
    codes = whole.codes[at // 16 * per:][:part.codes.numel()]
    full = part.rows // 16 * per                                            # what fills up the last 16 is other rows there
    assert torch.equal(codes[:full], part.codes[:full])
    assert torch.equal(whole.scale[at:at + part.rows], part.scale)


def test_coding_and_product(S):  # noqa: F811
    from paper_2410_13056_amd import binding as B
    ws, X = B.Workspace(DEV), _randn(1, MOST, 5, dtype=torch.float16)
    X[MOST - 1, 3], status = float("inf"), torch.zeros(1, dtype=torch.int32, device=DEV)
    rows, w = S.int8_rows(X, status=status), S.prepare_int8(_randn(2, 3, 5))
    assert status.item() == B.STATUS_NONFINITE
    Y, Z = S.int8_product(w, X, ws), S.int8_product(w, rows, ws, bias=_randn(3, 3))
    for at in range(0, MOST, PART):
        x = X[at:at + PART]
        _same_codes(rows, S.int8_rows(x), at)
        assert torch.equal(Y[at:at + PART], S.int8_product(w, x, ws))
        assert torch.equal(Z[at:at + PART], S.int8_product(w, S.int8_rows(x), ws, bias=_randn(3, 3)))


def test_weights(S):  # noqa: F811
    W = _randn(1, MOST, 5, dtype=torch.bfloat16)
    whole = S.prepare_int8(W)
    for at in (0, 2 * PART - 32, 2 * PART, 14 * PART, 16 * PART - 48):
        part = S.prepare_int8(W[at:at + 4000])
        full = part.d_out // 16 * 16 * 128
        assert torch.equal(whole.codes[at * 128:][:full], part.codes[:full]) and torch.equal(whole.scale[at:at + 4000], part.scale)


def test_two_weights(S):  # noqa: F811
    n = 4 * PART + 40
    G, U = _randn(1, n, 5, dtype=torch.float16), _randn(2, n, 5, dtype=torch.float16)
    whole = S.prepare_int8_gated(G, U)
    for at in (0, 2 * PART - 32, 2 * PART, 4 * PART - 16, 4 * PART, n - 40):
        part = S.prepare_int8_gated(G[at:at + 4000], U[at:at + 4000])
        full = part.d_out // 16 * 32
        assert torch.equal(whole.codes[at * 256:][:full * 128], part.codes[:full * 128])
        assert torch.equal(whole.scale[at * 2:][:full], part.scale[:full])


def test_norm_in_8_bits(S):  # noqa: F811
    X, A = _randn(1, MOST, 5, dtype=torch.float16), _randn(2, MOST, 5)
    rows, s = S.rms_norm(X, _randn(3, 5), add=A, coded=True)
    for at in range(0, MOST, PART):
        part, t = S.rms_norm(X[at:at + PART], _randn(3, 5), add=A[at:at + PART], coded=True)
        _same_codes(rows, part, at)
        assert torch.equal(s[at:at + PART], t)


def test_norm(S):  # noqa: F811
    """16 wavefronts a row, 2^22 rows and some, in place."""
    m, d, block = (1 << 22) + 100, 4097, 1 << 16
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB of free memory")
    one = _randn(1, block, d, dtype=torch.float16)
    X = torch.empty((m, d), dtype=torch.float16, device=DEV)
    for at in range(0, m, block):
        X[at:at + block] = one[:m - at]
    X[-1] = one[7]
    want, last = S.rms_norm(one, _randn(2, d)), S.rms_norm(one[7:8], _randn(2, d))
    S.rms_norm(X, _randn(2, d), out=X)
    assert torch.equal(X[-1:], last)
    X[-1] = want[(m - 1) % block]
    for at in range(0, m, block):
        assert torch.equal(X[at:at + block], want[:m - at])
