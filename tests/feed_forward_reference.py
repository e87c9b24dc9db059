"""Plain forms of the feed-forward operators on the CPU, in 64 bits, each with a bound on what fp32 arithmetic in the
documented order may be off by.  A half step of fp32 is 2^-24 of the value."""
import numpy as np
import torch
from scipy import special

import serving_reference as R

F = np.float32
HALF = 2.0 ** -24
ROUND = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINIEST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
ACTS = [None, "silu", "gelu", "gelu_tanh", "relu"]


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def act(v, name):
    """The activation of 64-bit v, and the relative error that fp32 may give it.  v / (1 + e^-u): the exponential's step (2
    halves) and the rounding of its factor, the sum's, the reciprocal's step and the product's, 8 in all with one to spare.  u
    of GELU_TANH is off by 6 halves of itself (a cube's three products, a sum, a product, the constant), which moves the quotient
    by that times u (1 - quotient).  GELU: erfc's own 16 halves, the halving's and the product's, and an argument off by 2,
    which moves the distribution by its density over itself."""
    if name is None or name == "relu":
        return (v if name is None else np.where(v < 0, 0.0, v)), np.zeros_like(v)
    if name == "silu":
        return v * special.expit(v), np.full_like(v, 8 * HALF)
    if name == "gelu":
        c = np.clip(v, -200, 200)
        slope = np.exp(-c * c / 2 - special.log_ndtr(c)) / np.sqrt(2 * np.pi)
        return v * special.ndtr(v), (20 + 2 * np.abs(c) * slope) * HALF
    u = np.sqrt(8 / np.pi) * (v + 0.044715 * v ** 3)
    return v * special.expit(u), (8 + 6 * np.abs(u) * special.expit(-u)) * HALF


def finish(p, off, bias=None, name=None, times=None, times_off=0.0, times_bias=None, residual=None):
    """act(p + bias) * (times + times_bias) + residual in 64 bits, and a bound, where p is off by `off` and times by `times_off`.
    No slope of the activations is above 1.13.  2^-118 and the second factor's share of it: results below the smallest numbers."""
    z, ez = p, off
    if bias is not None:
        z = p + bias
        ez = off + HALF * np.abs(z)
    v, rel = act(z, name)
    e = (1.13 if name else 1.0) * ez + rel * np.abs(v) + (2.0 ** -118 if name else 0)
    if times is not None:
        u, eu = times, times_off
        if times_bias is not None:
            u = times + times_bias
            eu = times_off + HALF * np.abs(u)
        e = e * np.abs(u) + np.abs(v) * eu + e * eu + HALF * np.abs(v * u)
        v = v * u
    if residual is not None:
        v = v + residual
        e = e + HALF * np.abs(v)
    return v, e


def check(got, want, bound):
    """got is want within the bound and its own type's half step."""
    g = got.double().cpu().numpy()
    assert g.shape == want.shape
    off = np.abs(g - want)
    room = bound * (1 + ROUND[got.dtype]) + np.abs(want) * ROUND[got.dtype] + TINIEST[got.dtype] + 4 * HALF * bound
    assert (off <= room).all(), (off - room).max()


def product(X, W):
    """The scaled sums in 64 bits, and their bound: a rounding of the sum and two of the products."""
    cx, sx = R.rows_in_8_bits(R.as_f32(X))
    cw, sw = R.rows_in_8_bits(R.as_f32(W))
    p = (cx.astype(np.float64) @ cw.T.astype(np.float64)) * sx[:, None].astype(np.float64) * sw
    return p, 4 * HALF * np.abs(p)


def norm(X, add, weight, eps, sum_dtype):
    """(y in fp32, s as a tensor of `sum_dtype`), operation by operation."""
    x = torch.from_numpy(R.as_f32(X))
    if add is not None:
        x = x + torch.from_numpy(R.as_f32(add))
    s = x if sum_dtype is None else x.to(sum_dtype)
    v = s.float().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        q = np.square(v.astype(np.float64)).sum(1, keepdims=True)
        r = (1.0 / np.sqrt(q / v.shape[1] + eps)).astype(F)
        y = v * r
        if weight is not None:
            y = y * R.as_f32(weight)
    return y, s


def coded(rows):
    """(codes [rows, dim], scales) out of an Int8Rows."""
    torch.cuda.synchronize()
    codes, below, beyond = R.weight_codes(rows.codes.cpu().numpy(), rows.rows, rows.dim)
    assert not below.any() and not beyond.any()
    return codes, rows.scale.cpu().numpy()
