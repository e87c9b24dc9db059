"""Attention over the paged cache where device data and the host's bounds disagree: what is left out is flagged, and
all else is what the call says it is."""
import numpy as np
import pytest
import torch

import serving_reference as R
import test_gpu_kv_attention as A

pytestmark = pytest.mark.gpu

DEV = "cuda"
# roundings of FP16 outputs relative to the largest value, logits of order one: the weights' 2^-11, the output's 2^-11, the
# query's 2^-16 of logits that it changes by at most `reach` (below 2^3 here) times that, twice
CLOSE = 2.0 ** -10 + 2.0 ** -11


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _call(S, s, Q, cu, lengths, max_rows, max_length, **kw):
    """Output on top of 5s, and the status."""
    from paper_2410_13056_amd import binding as B
    status, out = torch.zeros(1, dtype=torch.int32, device=DEV), torch.full_like(Q, 5.0)
    S.kv_attention(s.cache, Q, s.table, A._i32(lengths), A._i32(cu), max_rows, max_length, B.Workspace(DEV), out=out, status=status, **kw)
    torch.cuda.synchronize()
    return out, status.item()


def _tokens(s, i, n):
    return [c[s.order[i, :-(-n // s.page)]].transpose(0, 2, 1, 3).reshape(-1, c.shape[1], s.dim)[:n] for c in s.dense()]


def _near(got, want, v):
    off = np.abs(got.double().cpu().numpy() - want).max()
    assert off <= CLOSE * np.abs(v).max(), off


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("most", [1, 3, 100])
@pytest.mark.parametrize("beside", [1, 2])
def test_more_rows_than_the_bound_under_a_window(S, causal, most, beside):
    """A sequence that names 4000 rows more than the host's bound sees more units in its window than the host counts with;
    its first rows and the sequences behind it are done all the same."""
    from paper_2410_13056_amd import binding as B
    window, tokens = 2048, [6100] + [3000] * beside
    s = A.Setup(S, tokens, 1, 64, 32, 11)
    cu = [0, 4000] + [4000 + (i + 1) * most for i in range(beside)]
    Q = torch.randn((cu[-1], 2, 64), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).half() * 0.25
    out, status = _call(S, s, Q, cu, tokens, most, max(tokens), window=window, causal=causal)
    assert status == B.STATUS_RANGE and (out[most:4000] == 5).all()
    q = R.as_f32(Q).astype(np.float64)
    k, v = _tokens(s, 0, 6100)
    for row in {0, most - 1}:
        p = 2100 + row
        at = slice(max(0, p - window + 1), p + 1 if causal else 6100)
        _near(out[row], R.attention(q[row:row + 1], k[at], v[at], 0.125, False, 0)[0][0], v)
    for i in range(beside):
        k, v = _tokens(s, i + 1, 3000)
        a, b = cu[i + 1], cu[i + 2]
        _near(out[a:b], R.attention(q[a:b], k, v, 0.125, causal, window)[0], v)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 40, 70, 4000])
@pytest.mark.parametrize("rows", [1, 20, 70])
def test_tokens_that_are_left_out_do_not_move_the_rows(S, rows, window, causal):
    """A sequence of 300 tokens under bounds of 200 and 250, and of a table that ends at 256: its rows are the tokens
    300 - rows .. 299 all the same, turned and masked as such."""
    from paper_2410_13056_amd import binding as B
    s = A.Setup(S, [300], 1, 64, 32, 4)
    rotation = S.make_rotation(300, 64, device=DEV)
    Q = torch.randn((rows, 2, 64), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).half() * 0.25
    pos = 300 - rows + np.arange(rows)
    q = R.turn(R.as_f32(Q), pos, R.as_f32(rotation.cos), R.as_f32(rotation.sin), False).astype(np.float64)
    whole = s.table
    for bound, pages in ((200, 10), (250, 10), (300, 8)):
        s.table = whole[:, :pages].contiguous()
        left = min(bound, pages * 32)
        out, status = _call(S, s, Q, [0, rows], [300], rows, bound, rotation=rotation, causal=causal, window=window)
        assert status == B.STATUS_RANGE
        k, v = _tokens(s, 0, left)
        for r in range(rows):
            lo, hi = max(0, pos[r] - window + 1) if window else 0, min(left, pos[r] + 1) if causal else left
            if lo >= hi:
                assert (out[r] == 0).all()
            else:
                _near(out[r], R.attention(q[r:r + 1], k[lo:hi], v[lo:hi], 0.125, False, 0)[0][0], v)


@pytest.mark.parametrize("seqs", [1, 70])
def test_calls_without_room_for_rows_that_are_named_are_flagged(S, seqs):
    from paper_2410_13056_amd import binding as B
    s = A.Setup(S, [40] * seqs, 2, 64, 32, 3)
    none, one = [0] * (seqs + 1), [0] * seqs + [1]
    Q = torch.randn((1, 4, 64), device=DEV).half()
    for cu, flag in ((none, 0), (one, B.STATUS_RANGE)):
        for q, most in ((Q, 0), (Q[:0], 0), (Q[:0], 1)):
            out, status = _call(S, s, q, cu, [40] * seqs, most, 40)
            assert status == flag and (out == 5).all()
        K, held = torch.randn((1, 2, 64), device=DEV), A._i32([3] * seqs)
        for x, table in ((K[:0], s.table), (K, s.table[:, :0].contiguous())):
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            S.kv_append(s.cache, x, x, table, held, A._i32(cu), status=status)
            torch.cuda.synchronize()
            assert status.item() == flag
            status.zero_()
            B.kv_read(s.cache._view, table, held, A._i32(cu), x, x.clone(), status)
            torch.cuda.synchronize()
            assert status.item() == flag
