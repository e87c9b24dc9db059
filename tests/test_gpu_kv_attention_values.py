"""Attention over the paged cache where the values' sizes decide: near the top of a type's range, and of pages whose
scales lie many orders apart, judged row by row."""
import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("dim", [32, 40, 64, 96, 160])
@pytest.mark.parametrize("rows", [1, 60])
def test_parts_of_large_values_are_added_once(S, dim, rows):
    """700 tokens of 2^111 with weights alike: the sum 2^7 * 700 * 2^111 that the parts are added to is below 2^128, twice as
    much is not.  Rounded on the way: weights of 1 not at all, the scale and the output's quotient in fp32 (2^-22 in all)
    and the output to bfloat16."""
    s = A.Bounded(S, [700], 1, dim, 32, dim)
    s.cache.v.fill_(255)
    s.cache.v_scale.fill_(2.0 ** 111 / 127)
    Q = torch.randn((rows, 2, dim), device=DEV).bfloat16()
    out = s.run(Q, [rows], softmax_scale=0.0)
    torch.cuda.synchronize()
    off = np.abs(out.double().cpu().numpy() / 2.0 ** 111 - 1)
    assert (off <= 2.0 ** -8 + 2.0 ** -22).all(), off.max()


def _row_by_row(s, Q, window, out):
    """One sequence, one key / value head, against 64 bits, every element held to its own row's values.  With a_t = w_t v_t / sum w:
    a weight is off by 2^-11 of itself (FP16) or, once that is more, by 2^-25 of where the largest a row has is above 2^7;
    an element of the query by 2^-16 of the row's largest, so a logit by `reach` 2^-16 and a weight's share by expm1(2 that);
    the rest are fp32 roundings and the output's own."""
    got = s.run(Q, [Q.shape[0]], window=window, out_dtype=out)
    again = s.run(Q, [Q.shape[0]], window=window, out_dtype=out)
    torch.cuda.synchronize()
    assert torch.equal(got, again)
    got = got.double().cpu().numpy()
    k, v = (c[s.order[0, :-(-s.tokens[0] // s.page)]].transpose(0, 2, 1, 3).reshape(-1, s.dim)[:s.tokens[0]] for c in s.dense())
    scale = np.repeat(s.cache.v_scale.double().cpu().numpy()[s.order[0, :-(-s.tokens[0] // s.page)], 0], s.page)[:s.tokens[0]]
    t, rows, q = s.tokens[0], Q.shape[0], Q.double().cpu().numpy()
    pos, at = t - rows + np.arange(rows), np.arange(t)
    seen = (at[None] <= pos[:, None]) & (at[None] > pos[:, None] - (window or t + 1))
    judged = 0
    for h in range(Q.shape[1]):
        logits = np.where(seen, q[:, h] @ k.T * s.dim ** -0.5, -np.inf)
        w = np.exp(logits - logits.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        want, size, most = w @ v, w @ np.abs(v), (w * scale).max(1, keepdims=True)
        reach = s.dim ** -0.5 * np.abs(k).sum(1).max() * np.abs(q[:, h]).max(1, keepdims=True)
        u, least, top = (2.0 ** -11, 2.0 ** -24, 60000.0) if out == torch.float16 else (2.0 ** -8, 0.0, 3e38)
        bound = size * (np.expm1(2 * reach * 2.0 ** -16) + 2.0 ** -11 + 2.0 ** -18) + t * 127 * 2.0 ** -32 * most + u * np.abs(want) + least
        ok = np.abs(want).max(1) < top
        off = np.abs(got[:, h] - want)
        assert (off[ok] <= bound[ok]).all(), (h, (off[ok] / bound[ok]).max())
        judged += int(ok.sum())
    return judged


@pytest.mark.parametrize("rows", [1, 3, 48, 150])
@pytest.mark.parametrize("above", [0, 20, 24, 28, 32, 33, 40, 62, 90])
def test_pages_far_above_that_a_row_hardly_attends_to(S, rows, above):
    # the first page's values are 2^above of the others, its weights 2^-(above + 60)
    s = A.Setup(S, [256], 1, 64, 32, above + rows, size=1 / 400)
    first = int(s.order[0, 0])
    s.cache.k[first], s.cache.k_scale[first] = 1, (above + 60) * np.log(2) / 8 / 127
    s.cache.v_scale[first] *= 2.0 ** above
    g = torch.Generator(device=DEV).manual_seed(above)
    Q = (1 + torch.randn((rows, 2, 64), generator=g, device=DEV) * 0.01).half()
    for out in (torch.float16, torch.bfloat16):
        assert _row_by_row(s, Q, 0, out) == 2 * rows


@pytest.mark.parametrize("rows", [1, 48, 150])
@pytest.mark.parametrize("above", [24, 32, 40, 90])
@pytest.mark.parametrize("window,page", [(64, 1), (64, 4), (64, 6), (64, 7), (0, 6), (0, 7)])
def test_pages_far_above_that_a_row_does_not_see(S, rows, above, window, page):
    # rows beside it in the tile do see the page
    s = A.Setup(S, [256], 1, 64, 32, above + rows)
    s.cache.v_scale[int(s.order[0, page])] *= 2.0 ** above
    g = torch.Generator(device=DEV).manual_seed(above)
    Q = torch.randn((rows, 1, 64), generator=g, device=DEV).half()
    _row_by_row(s, Q, window, torch.float16)
    assert _row_by_row(s, Q, window, torch.bfloat16) == rows


@pytest.mark.parametrize("rows", [1, 40, 150])
@pytest.mark.parametrize("seed", range(4))
def test_scales_of_any_size_row_by_row(S, rows, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    for kind, tokens in ((A.Setup, 700), (A.Bounded, 700)):                 # in one part, and joined
        s = kind(S, [tokens], 1, 64, 32, seed)
        s.cache.v_scale.mul_(torch.exp(torch.randn(s.cache.v_scale.shape, device=DEV, generator=g) * 15))
        s.cache.k_scale.mul_(torch.exp(torch.randn(s.cache.k_scale.shape, device=DEV, generator=g)))
        Q = torch.randn((rows, 1, 64), generator=g, device=DEV).half()
        assert _row_by_row(s, Q, 200 * (seed % 2), torch.bfloat16) == rows


def test_results_do_not_depend_on_the_rows_beside(S):
    s = A.Setup(S, [256], 1, 64, 32, 5)
    for page, by in ((0, 2.0 ** 30), (5, 2.0 ** -35), (7, 2.0 ** 50)):
        s.cache.v_scale[int(s.order[0, page])] *= by * 1.3
    Q = torch.randn((40, 1, 64), device=DEV).bfloat16()
    both = s.run(Q, [40])
    Q[:20], Q[30:] = Q[:20] * 3, -Q[30:]
    assert torch.equal(s.run(Q, [40])[20:30], both[20:30])
