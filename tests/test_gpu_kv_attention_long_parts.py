"""Attention whose parts are longer than the pages that a wavefront takes the numbers and scales of at a time: 64 units
of 32 tokens for many rows, 64 a wavefront (256 a workgroup) for few.  A part has at least as many units as
units * tiles / 512 (256 where a wavefront has three tiles), so enough tiles make it the whole sequence.  Sequences share
their pages, each in an order of its own, with scales that differ by page; some rows are checked."""
import numpy as np
import pytest
import torch

import serving_reference as R
import test_gpu_kv_attention as A

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _check_some(S, seqs, tokens, rows, kv, group, dim, page, causal, window, check, seed):
    """`check`: (sequence, row) pairs.  Bounds as in the tests of attention, the query off by 2^-16."""
    s = A.Setup(S, [tokens], kv, dim, page, seed, spread=1.0)
    n = -(-tokens // page)
    rng = np.random.default_rng(seed)
    order = np.stack([rng.permutation(s.order[0, :n]) for _ in range(seqs)])
    g = torch.Generator(device=DEV).manual_seed(seed)
    Q = torch.randn((seqs * rows, kv * group, dim), generator=g, device=DEV).half() * 0.5
    cu, lens, table = A._i32([i * rows for i in range(seqs + 1)]), A._i32([tokens] * seqs), A._i32(order.tolist())
    out = S.kv_attention(s.cache, Q, table, lens, cu, rows, tokens, causal=causal, window=window)
    assert torch.equal(out, S.kv_attention(s.cache, Q, table, lens, cu, rows, tokens, causal=causal, window=window))
    k, v = s.dense()
    for i, row in check:
        p, at = tokens - rows + row, i * rows + row
        lo, hi = max(0, p - window + 1) if window else 0, p + 1 if causal else tokens
        kk, vv = (c[order[i]].transpose(0, 2, 1, 3).reshape(-1, kv, dim)[lo:hi] for c in (k, v))
        want, reach = R.attention(R.as_f32(Q[at:at + 1]).astype(np.float64), kk, vv, dim ** -0.5, False, 0)
        off = np.abs(out[at].double().cpu().numpy() - want[0])
        assert (off <= np.abs(vv).max() * (2 * np.expm1(2 * reach * 2.0 ** -16) + 2.0 ** -11) + 2.0 ** -11 * np.abs(want[0]) + 2.0 ** -24).all(), \
            (i, row, off.max())


@pytest.mark.parametrize("units", [63, 64, 65, 128, 129, 193])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 2048)])
@pytest.mark.parametrize("dim,page", [(32, 64), (128, 32), (192, 32)])
def test_many_rows(S, units, causal, window, dim, page):
    # 8 heads * 66 tiles of 64 columns, so that a part is a sequence's whole; of 128 dims from 95 units on 8 * 22 tiles of 192, whose
    # parts are half as long
    tokens = units * 32 - 5
    _check_some(S, 1, tokens, 528, 8, 8, dim, page, causal, window, [(0, r) for r in (0, 1, 7, 8, 300, 527)], units)


@pytest.mark.parametrize("units", [64, 65, 129])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_of_three_tiles_a_wavefront(S, units, causal):
    rows = min(units * 32 - 5, 50000 // units * 192 // 64 + 24)          # 50000 units of tiles of 192 columns
    _check_some(S, max(1, (50000 // units * 192 // 64 + 24) // rows + 1), units * 32 - 5, rows, 8, 8, 128, 32, causal, 0,
                [(0, r) for r in (0, 23, rows - 1)], units)


@pytest.mark.parametrize("tokens,rows", [(300 * 32, 256), (200 * 64 + 3, 300)])
def test_many_rows_joined_of_long_parts(S, tokens, rows):
    _check_some(S, 1, tokens, rows, 8, 8, 64, 64, True, 0, [(0, r) for r in (0, 100, rows - 1)], rows)


@pytest.mark.parametrize("units", [255, 256, 257, 300, 511, 513])
@pytest.mark.parametrize("group,dim", [(1, 32), (8, 64), (20, 128), (48, 32)])
def test_few_rows(S, units, group, dim):
    # 512 tiles of a sequence and head, a row each
    _check_some(S, 128, units * 32 - 9, 1, 4, group, dim, 64 if units % 2 else 32, True, 0, [(i, 0) for i in (0, 63, 64, 127)], units)


@pytest.mark.parametrize("rows,window", [(3, 0), (3, 9000), (6, 0)])
def test_few_rows_of_drafts(S, rows, window):
    _check_some(S, 128, 400 * 32 + 1, rows, 4, 5, 64, 32, True, window, [(i, r) for i in (0, 127) for r in (0, rows - 1)], rows)
