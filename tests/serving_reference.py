"""Plain forms of 8-bit serving on the CPU: codes and scales operation by operation in fp32 (so that they can be
compared bit for bit), sums and softmax in 64 bits."""
import numpy as np

F = np.float32
TINY = F(2.0 ** -126)


def as_f32(t):
    """A torch tensor of any of the three types as numpy fp32 (exact)."""
    return t.detach().float().cpu().numpy()


def scale_of(x, axes):
    a = np.abs(x)
    a = np.where(np.isfinite(a), a, F(0))
    return np.maximum(a.max(axis=axes, initial=F(0)) / F(127), TINY).astype(F)


def codes_of(x, inv):
    with np.errstate(invalid="ignore", over="ignore"):
        t = np.clip(x * inv, F(-127), F(127))
    return np.rint(np.where(np.isnan(x), F(0), t)).astype(np.int32)


def rows_in_8_bits(x):
    """Codes [n, d] and scales [n]."""
    s = scale_of(x, 1)
    return codes_of(x, (F(1) / s)[:, None]), s


def weight_codes(stored, d_out, d_in):
    """Codes [d_out, d_in] out of the prepared weight's pieces, and what the rest of it holds."""
    deep, groups = (d_in + 127) // 128 * 2, (d_out + 15) // 16
    x = stored.reshape(groups, deep, 4, 16, 16).transpose(0, 3, 1, 2, 4).reshape(groups * 16, deep * 64)
    return x[:d_out, :d_in], x[d_out:], x[:, d_in:]


def turn(x, positions, cos, sin, interleaved):
    """Rows [n, heads, dim] turned by position; every product and sum rounded to fp32."""
    if cos is None:
        return x.copy()
    half = cos.shape[1]
    ia, ib = (np.arange(half) * 2, np.arange(half) * 2 + 1) if interleaved else (np.arange(half), np.arange(half) + half)
    at = np.minimum(positions, cos.shape[0] - 1)
    c, s = cos[at][:, None], sin[at][:, None]
    a, b, y = x[..., ia], x[..., ib], x.copy()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


class Pages:
    """A cache as codes [pages, heads, tokens, dims] and scales [pages, heads], one of keys or values."""

    def __init__(self, n_pages, heads, page, dim):
        self.codes = np.zeros((n_pages, heads, page, dim), np.int32)
        self.scale = np.zeros((n_pages, heads), F)
        self.page = page

    def append(self, x, table, held):
        """Tokens x [n, heads, dim] of one sequence behind `held`; `table` its pages."""
        done = 0
        while done < len(x):
            at = held + done
            p, off = table[at // self.page], at % self.page
            n = min(self.page - off, len(x) - done)
            new = x[done:done + n]
            old = self.scale[p] if off else np.zeros_like(self.scale[p])
            scale = np.maximum(old, scale_of(new, (0, 2)))
            inv = F(1) / scale
            again = np.rint(self.codes[p, :, :off].astype(F) * (old * inv)[:, None, None]).astype(np.int32)
            grown = (scale != old)[:, None, None]
            self.codes[p, :, :off] = np.where(grown, again, self.codes[p, :, :off])
            self.codes[p, :, off:off + n] = codes_of(new, inv[None, :, None]).transpose(1, 0, 2)
            self.scale[p] = scale
            done += n


def page_codes(stored, keys, page, dim):
    """Codes [pages, heads, tokens, dims (whole pieces)] out of the stored bytes [pages, heads, bytes]."""
    c = (dim + 31) // 32
    x = stored.reshape(*stored.shape[:2], page // 32, c, 4, 16, 2, 8).astype(np.int32) - 128
    if keys:                                    # [g][t][h][j]: token 16 h + t, dim 8 g + j
        x = x.transpose(0, 1, 2, 6, 5, 3, 4, 7)
    else:                                       # token 16 (j / 4) + 4 g + j % 4, dim 16 h + t
        x = x.reshape(*stored.shape[:2], page // 32, c, 4, 16, 2, 2, 4).transpose(0, 1, 2, 7, 4, 8, 3, 6, 5)
    return x.reshape(*stored.shape[:2], page, c * 32)


def attention(q, k, v, scale, causal, window):
    """q [rows, q_heads, dim], k and v [tokens, kv_heads, dim], in 64 bits: O, and the largest change of a logit when
    every |q| changes by its row's largest magnitude (for tolerances)."""
    rows, heads, dim = q.shape
    t, kv, _ = k.shape
    out, reach = np.zeros((rows, heads, dim)), 0.0
    if t == 0 or rows == 0:
        return out, reach
    group = heads // kv
    pos = t - rows + np.arange(rows)
    at = np.arange(t)
    seen = np.ones((rows, t), bool)
    if causal:
        seen &= at[None] <= pos[:, None]
    if window:
        seen &= at[None] > pos[:, None] - window
    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(heads):
            kh, vh = k[:, h // group], v[:, h // group]
            logits = np.where(seen, (q[:, h] @ kh.T) * scale, -np.inf)
            top = logits.max(1, keepdims=True)
            w = np.exp(logits - np.where(np.isneginf(top), 0, top))
            total = w.sum(1, keepdims=True)
            out[:, h] = (w @ vh) / np.where(total == 0, 1, total)
            reach = max(reach, float(np.abs(scale) * np.abs(kh).sum(1).max() * np.nan_to_num(np.abs(q[:, h])).max()))
    return out, reach
