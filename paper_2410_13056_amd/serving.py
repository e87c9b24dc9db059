"""Serving in 8 bits: what a decoder layer needs beside the products with the mixed-precision
weights (`pipeline.lut_matvec`, `pipeline.group_products`).

* `prepare_int8`, `int8_product`: a linear layer in 8-bit integers, for layers that are not to go below
  8 bits and for prompts, where multiplications bound the product; bias, activation and residual on the way out;
* `prepare_int8_gated`, `int8_gated_product`: the two projections of a gated feed-forward part in one pass;
* `rms_norm`: the norm before a part of the layer, with the sum of the residual stream, as values or as rows in 8
  bits (`Int8Rows`, `int8_rows`), which one coding hands to all products that share the input;
* `epilogue`: what may follow a product, for products in mixed precision;
* `feed_forward_block`: norm, gated projections, output projection and residual, as a decoder layer runs them;
* `KvCache`, `kv_append`, `kv_read`: keys and values in pages of 8-bit codes, keys turned by position on the way in;
* `kv_attention`: attention over the cache, for single tokens, drafts and chunks of prompts;
* `attention_block`: products, cache and attention together, as a decoder layer's attention runs them.

Everything is enqueued on the current stream and nothing synchronises; there is no gradient, since
codes have none.  `status` ([1] int32, cleared by the caller) collects the flags of `binding.STATUS_*`: codes have no NaN
and no infinity (they become 0 and +-127 codes), so without it such an input goes unnoticed.
"""
from __future__ import annotations

import dataclasses
import functools
from typing import Callable, Optional, Sequence, Tuple, Union

import torch

from . import binding as B
from . import pipeline as P


class _Kept:
    """An object whose fields calls are handed in a form that `_make` gives; that is made once, and again after a field is
    assigned.  Copies make their own."""

    def __post_init__(self):
        self._args                          # refuses fields that do not fit

    @functools.cached_property
    def _args(self):
        return self._make()

    def __setattr__(self, name, value):
        self.__dict__[name] = value
        self.__dict__.pop("_args", None)

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k != "_args"}


# ---- products --------------------------------------------------------------------------------

@dataclasses.dataclass
class Int8Weight(_Kept):
    """A linear layer as `int8_product` reads it (device tensors)."""
    d_in: int
    d_out: int
    codes: torch.Tensor     # int8, in the order of the matrix instruction's operands
    scale: torch.Tensor     # [d_out] fp32

    def _make(self) -> B.Int8ProductCall:
        return B.Int8ProductCall(self.d_in, self.d_out, self.codes, self.scale)


def prepare_int8(W: torch.Tensor, status: Optional[torch.Tensor] = None) -> Int8Weight:
    """A weight [d_out, d_in] (the framework layout) in 8 bits with a scale per output channel."""
    d_out, d_in = W.shape
    codes = torch.empty(B.int8_weight_bytes(d_out, d_in), dtype=torch.int8, device=W.device)
    scale = torch.empty(d_out, dtype=torch.float32, device=W.device)
    B.int8_prepare(W, codes, scale, status)
    return Int8Weight(d_in, d_out, codes, scale)


@dataclasses.dataclass
class Int8Rows(_Kept):
    """Inputs [rows, dim] in 8 bits with a scale each, as the products read them (device tensors)."""
    rows: int
    dim: int
    codes: torch.Tensor     # int8, in the order of the matrix instruction's operands
    scale: torch.Tensor     # [rows] fp32

    def _make(self) -> B.Int8RowsView:
        return B.Int8RowsView(self.rows, self.dim, self.codes, self.scale)

    def __getattr__(self, name):
        """Codes and scales of rows that were made in one piece, when something asks for them: most only pass through."""
        if name in ("codes", "scale") and "_whole" in self.__dict__:
            whole, n = self.__dict__["_whole"], B.int8_weight_bytes(self.rows, self.dim)
            t = self.__dict__[name] = whole[:n] if name == "codes" else whole[n:].view(torch.float32)
            return t
        raise AttributeError(name)


def _empty_rows(like: torch.Tensor) -> Int8Rows:
    """Room for the rows of `like` in 8 bits."""
    rows, dim = like.shape
    nbytes = B.int8_weight_bytes(rows, dim)     # a multiple of 1 KB: the scales behind it are aligned
    whole = like.new_empty(nbytes + 4 * rows, dtype=torch.int8)
    made = Int8Rows.__new__(Int8Rows)           # without the checks of tensors that come from elsewhere
    made.__dict__.update(rows=rows, dim=dim, _whole=whole, _args=B.Int8RowsView.of_whole(rows, dim, whole, nbytes))
    return made


def int8_rows(X: torch.Tensor, out: Optional[Int8Rows] = None, status: Optional[torch.Tensor] = None) -> Int8Rows:
    """Inputs X [m, d_in] in 8 bits, coded once for all products that share them: these give what they give for X."""
    if out is None:
        out = _empty_rows(X)
    elif (out.rows, out.dim) != tuple(X.shape):
        raise ValueError("the rows in 8 bits must be of X's shape")
    B.int8_prepare(X, out.codes, out.scale, status)
    return out


Inputs = Union[torch.Tensor, Int8Rows]


def _output(X: Inputs, d_out: int, out_dtype: Optional[torch.dtype]) -> torch.Tensor:
    if isinstance(X, Int8Rows):
        return X._args.keep[0].new_empty((X.rows, d_out), dtype=out_dtype or torch.float16)
    return X.new_empty((X.shape[0], d_out)) if out_dtype is None else X.new_empty((X.shape[0], d_out), dtype=out_dtype)


def int8_product(w: Int8Weight, X: Inputs, ws: Optional[B.Workspace] = None,
                 out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                 activation: Optional[str] = None, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y [m, d_out] = act(X [m, d_in] times the weight + bias) + residual, X in 8 bits with a scale per token on the way, or
    already (`Int8Rows`).  `out_dtype` defaults to X's (float16 for rows in 8 bits).  `bias` [d_out]; `activation`
    "silu", "gelu", "gelu_tanh" or "relu"; `residual` [m, d_out], which may be `out` itself; each of its own type.  All of it
    is worked out in fp32 and rounded once."""
    made = out is None
    if made:
        out = _output(X, w.d_out, out_dtype)
    coded = isinstance(X, Int8Rows)
    if not coded and bias is None and activation is None and residual is None:
        w._args(X, out, ws or B.Workspace(X.device), status)
    else:
        w._args.job(X._args if coded else X, out, ws or B.Workspace(out.device), status, bias, None, activation, residual,
                    made)
    return out


@dataclasses.dataclass
class Int8GatedWeight(_Kept):
    """The two projections of a gated feed-forward part as `int8_gated_product` reads them (device tensors)."""
    d_in: int
    d_out: int              # of each
    codes: torch.Tensor     # int8, groups of 16 outputs of the gate and of the second factor in turn
    scale: torch.Tensor     # fp32, in that order

    def _make(self) -> B.Int8ProductCall:
        return B.Int8ProductCall(self.d_in, self.d_out, self.codes, self.scale, gated=True)


def prepare_int8_gated(W_gate: torch.Tensor, W_up: torch.Tensor, status: Optional[torch.Tensor] = None) -> Int8GatedWeight:
    """Two weights [d_out, d_in] of one type in 8 bits with a scale per output channel."""
    d_out, d_in = W_gate.shape
    rows = B.int8_gated_rows(d_out)
    codes = torch.empty(B.int8_weight_bytes(rows, d_in), dtype=torch.int8, device=W_gate.device)
    scale = torch.empty(rows, dtype=torch.float32, device=W_gate.device)
    B.int8_prepare_gated(W_gate, W_up, codes, scale, status)
    return Int8GatedWeight(d_in, d_out, codes, scale)


def int8_gated_product(w: Int8GatedWeight, X: Inputs, ws: Optional[B.Workspace] = None, activation: Optional[str] = "silu",
                       gate_bias: Optional[torch.Tensor] = None, up_bias: Optional[torch.Tensor] = None,
                       out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                       status: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """H [m, d_out] = act(X Wg' + gate_bias) * (X Wu' + up_bias) (+ residual): one pass over the inputs, neither projection in
    memory.  Otherwise as `int8_product`; the biases are of one type."""
    made = out is None
    if made:
        out = _output(X, w.d_out, out_dtype)
    w._args.job(X._args if isinstance(X, Int8Rows) else X, out, ws or B.Workspace(out.device), status, gate_bias, up_bias,
                activation, residual, made)
    return out


# ---- what stands between products --------------------------------------------------------------

def epilogue(Y: torch.Tensor, bias: Optional[torch.Tensor] = None, activation: Optional[str] = None,
             times: Optional[torch.Tensor] = None, times_bias: Optional[torch.Tensor] = None,
             residual: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
             out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """act(Y + bias) * (times + times_bias) + residual for the outputs Y [m, d] of a product in mixed precision; times and
    residual are [m, d], the biases [d], each of its own type.  `out_dtype` defaults to Y's; `out` may be Y, times or residual.
    Asked for nothing, the answer is Y itself, as with `Tensor.to`."""
    made = out is None
    if made and bias is activation is times is times_bias is residual is None and out_dtype in (None, Y.dtype):
        B.check_matrix(Y)
        return Y
    if made:
        out = torch.empty_like(Y, dtype=out_dtype)
    B.epilogue(Y, out, bias, activation, times, times_bias, residual, made)
    return out


def rms_norm(X: torch.Tensor, weight: Optional[torch.Tensor] = None, eps: float = 1e-6, add: Optional[torch.Tensor] = None,
             coded: bool = False, out: Optional[Inputs] = None, out_dtype: Optional[torch.dtype] = None,
             sum_out: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """s / sqrt(mean(s^2) + eps) * weight along the rows of s = X [m, d], or of s = X + add; the weight [d] may be None.
    `coded`: as `Int8Rows` for the products that follow, else of `out_dtype`, by default X's.  With `add` the answer is (norm, s),
    s of X's type unless `sum_out` says otherwise, which may be X or `add` itself; the norm is that of s as rounded."""
    made, sum_made = out is None, add is not None and sum_out is None
    if made:
        out = _empty_rows(X) if coded else torch.empty_like(X, dtype=out_dtype)
    if sum_made:
        sum_out = torch.empty_like(X)
    B.rms_norm(X, weight, eps, out._args if isinstance(out, Int8Rows) else out, add, sum_out, status, made, sum_made)
    return out if add is None else (out, sum_out)


@dataclasses.dataclass
class RmsNorm:
    """A norm's weight [d] (None: ones) and epsilon, as `rms_norm` takes them."""
    weight: Optional[torch.Tensor] = None
    eps: float = 1e-6


# ---- the cache -------------------------------------------------------------------------------

@dataclasses.dataclass
class Rotation(_Kept):
    """Turning by position: tables [positions, dims / 2] of the pairs' cosines and sines; the pairs are (j, j + dims / 2)
    of a head's first `dims` dims, or (2 j, 2 j + 1) where `interleaved`."""
    cos: torch.Tensor
    sin: torch.Tensor
    interleaved: bool = False

    def _make(self) -> B.RotationView:
        return B.rotation_view(self.cos, self.sin, self.interleaved)


def make_rotation(positions: int, dims: int, base: float = 10000.0, interleaved: bool = False,
                  device="cuda") -> Rotation:
    """The tables of angle p * base^(-2 j / dims)."""
    if dims < 2 or dims % 2 or positions < 1:
        raise ValueError("dims are turned in pairs: an even number of them; there is at least one position")
    half = dims // 2
    freq = torch.pow(float(base), -torch.arange(half, dtype=torch.float64) / half)
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * freq
    return Rotation(angle.cos().float().to(device), angle.sin().float().to(device), interleaved)


@dataclasses.dataclass
class KvCache(_Kept):
    """Keys and values in pages of `page` tokens, 8 bits a value, a scale per page and head (device tensors).
    Which page belongs to which sequence is the caller's: every call takes a table of them."""
    k: torch.Tensor         # uint8 [n_pages, kv_heads, kv_page_bytes(head_dim, page)]: code + 128
    v: torch.Tensor
    k_scale: torch.Tensor   # fp32 [n_pages, kv_heads]
    v_scale: torch.Tensor
    page: int
    head_dim: int

    def _make(self) -> B.KvCacheView:
        return B.kv_cache_view(self.k, self.v, self.k_scale, self.v_scale, self.page, self.head_dim)

    @property
    def _view(self) -> B.KvCacheView:
        return self._args

    @property
    def kv_heads(self) -> int:
        return self.k_scale.shape[1]


def make_cache(n_pages: int, kv_heads: int, head_dim: int, page: int = 64, device="cuda") -> KvCache:
    """An empty cache; nothing in it has to be cleared."""
    nbytes = B.kv_page_bytes(head_dim, page)
    if nbytes == 0:
        raise ValueError("head_dim is 1..256, a page 32..1024 tokens and a multiple of 32")
    codes = [torch.empty((n_pages, kv_heads, nbytes), dtype=torch.uint8, device=device) for _ in range(2)]
    scales = [torch.empty((n_pages, kv_heads), dtype=torch.float32, device=device) for _ in range(2)]
    return KvCache(codes[0], codes[1], scales[0], scales[1], page, head_dim)


def kv_append(cache: KvCache, K: torch.Tensor, V: torch.Tensor, page_table: torch.Tensor, held: torch.Tensor,
              cu_rows: torch.Tensor, rotation: Optional[Rotation] = None,
              status: Optional[torch.Tensor] = None) -> None:
    """Rows cu_rows[i] .. cu_rows[i+1]-1 of K and V [rows, kv_heads, head_dim] become the tokens held[i], held[i]+1,
    ... of sequence i, keys turned by `rotation` at their position.  `page_table` [n_seq, pages] int32 names the
    sequences' pages; `held` [n_seq] and `cu_rows` [n_seq + 1] are int32 too.  K and V may be views."""
    B.kv_append(cache._args, page_table, held, cu_rows, K, V, None if rotation is None else rotation._args, status)


def kv_read(cache: KvCache, page_table: torch.Tensor, first: torch.Tensor, cu_rows: torch.Tensor, n_rows: int,
            dtype: torch.dtype = torch.float16,
            status: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Keys and values [n_rows, kv_heads, head_dim] that the tokens first[i], first[i]+1, ... of each sequence stand
    for, cu_rows[i+1] - cu_rows[i] of them.  Rows that name no token of the cache are left as they come."""
    K = torch.empty((n_rows, cache.kv_heads, cache.head_dim), dtype=dtype, device=cache.k.device)
    V = torch.empty_like(K)
    B.kv_read(cache._args, page_table, first, cu_rows, K, V, status)
    return K, V


def kv_attention(cache: KvCache, Q: torch.Tensor, page_table: torch.Tensor, lengths: torch.Tensor,
                 cu_rows: torch.Tensor, max_rows: int, max_length: int, ws: Optional[B.Workspace] = None,
                 softmax_scale: Optional[float] = None, causal: bool = True, window: int = 0,
                 rotation: Optional[Rotation] = None, out: Optional[torch.Tensor] = None,
                 out_dtype: Optional[torch.dtype] = None, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of Q [rows, q_heads, head_dim] over the cache: rows cu_rows[i] .. cu_rows[i+1]-1 are the last tokens of
    sequence i, which has lengths[i].  `max_rows` and `max_length` bound both on the host.  A row sees the tokens up
    to its own (all of them unless `causal`), the last `window` of those where window > 0; one that sees none gives
    zeros.  `softmax_scale` defaults to head_dim^-0.5; the output is float16 or bfloat16, by default Q's type
    (float16 for float32)."""
    if out is None:
        out = torch.empty(Q.shape, dtype=out_dtype or (torch.float16 if Q.dtype == torch.float32 else Q.dtype),
                          device=Q.device)
    B.kv_attention(cache._args, page_table, lengths, cu_rows, Q, out, max_rows, max_length,
                   cache.head_dim ** -0.5 if softmax_scale is None else softmax_scale, ws or B.Workspace(Q.device), causal,
                   window, None if rotation is None else rotation._args, status)
    return out


# ---- a decoder layer's attention ---------------------------------------------------------------

Layer = Union[Int8Weight, P.Deployed, Callable[[torch.Tensor], torch.Tensor]]


def apply_layer(layer: Layer, X: Inputs, ws: B.Workspace, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """X [m, d_in] times a layer in whichever form it was prepared: 8-bit integers, the mixed-precision tables
    (fp32 out of FP16 in), or any function.  The last two carry a NaN or an infinity on into their outputs; 8-bit
    integers raise it in `status`, and take rows in 8 bits too."""
    if isinstance(layer, Int8Weight):
        return int8_product(layer, X, ws, out_dtype=torch.float32, status=status)
    if isinstance(layer, P.Deployed):
        return P.lut_matvec(layer, X.to(torch.float16), ws)
    return layer(X)


def _as_heads(Y: torch.Tensor, head_dim: int) -> torch.Tensor:
    """[rows, heads * head_dim], of no rows as well, as [rows, heads, head_dim] with unit stride along the dims."""
    Y = Y if Y.stride(1) == 1 else Y.contiguous()
    return Y.reshape(Y.shape[0], Y.shape[1] // head_dim, head_dim)


def _shared(X: torch.Tensor, layers, status: Optional[torch.Tensor]) -> Inputs:
    """What layers take that share the input X: in 8 bits if all of them are, coded once for all (one or two tokens code
    themselves within the products' launches)."""
    coded = X.shape[0] > 2 and all(isinstance(l, Int8Weight) for l in layers)
    return int8_rows(X, status=status) if coded else X


def _normed(X: torch.Tensor, norm: RmsNorm, layers, status: Optional[torch.Tensor],
            add: Optional[torch.Tensor] = None) -> Tuple[Sequence[Inputs], torch.Tensor]:
    """What each of the layers takes that share the norm of X (+ `add`), and that sum: in 8 bits if all of them are, coded once for
    all.  Else values: functions take X's type, the others too, or float16 where one of them is in mixed precision, which
    reads that."""
    mixed = functions = False
    for l in layers:
        if isinstance(l, P.Deployed):
            mixed = True
        elif not isinstance(l, (Int8Weight, Int8GatedWeight)):
            functions = True
    N = rms_norm(X, norm.weight, norm.eps, add, not (mixed or functions), out_dtype=torch.float16 if mixed else X.dtype, status=status)
    if add is not None:
        N, X = N
    if not (mixed and functions) or X.dtype == torch.float16:
        return [N] * len(layers), X
    own = rms_norm(X, norm.weight, norm.eps, status=status)
    return [N if isinstance(l, (Int8Weight, P.Deployed)) else own for l in layers], X


def attention_block(cache: KvCache, X: torch.Tensor, q: Layer, k: Layer, v: Layer, o: Layer, page_table: torch.Tensor,
                    held: torch.Tensor, lengths: torch.Tensor, cu_rows: torch.Tensor, max_rows: int,
                    max_length: int, ws: B.Workspace, rotation: Optional[Rotation] = None, causal: bool = True,
                    window: int = 0, status: Optional[torch.Tensor] = None,
                    attention_dtype: Optional[torch.dtype] = None, norm: Optional[RmsNorm] = None) -> torch.Tensor:
    """A decoder layer's attention for new tokens X [rows, hidden] of several sequences (see `kv_append`; lengths[i] =
    held[i] + the sequence's rows): the three projections, keys and values into the cache, attention over it, the
    output projection [rows, hidden].  The projections may be of different kinds, for instance queries and outputs in
    mixed precision and the short key and value layers in 8 bits.  `status` collects the flags of all of them.
    `attention_dtype`, float16 or bfloat16: what the attention hands to `o`.  By default bfloat16 for a bfloat16 X, whose
    values may pass float16's range, unless `o` is in mixed precision, which reads float16; else float16.
    `norm`: X is the residual stream, and the projections take its norm."""
    if attention_dtype is None:
        wide = X.dtype == torch.bfloat16 and not isinstance(o, P.Deployed)
        attention_dtype = torch.bfloat16 if wide else torch.float16
    Xs = [_shared(X, (q, k, v), status)] * 3 if norm is None else _normed(X, norm, (q, k, v), status)[0]
    Q, K, V = (_as_heads(apply_layer(layer, x, ws, status), cache.head_dim) for layer, x in zip((q, k, v), Xs))
    kv_append(cache, K, V, page_table, held, cu_rows, rotation, status)
    O = kv_attention(cache, Q, page_table, lengths, cu_rows, max_rows, max_length, ws, causal=causal, window=window,
                     rotation=rotation, out_dtype=attention_dtype, status=status)
    return apply_layer(o, O.flatten(1), ws, status)


# ---- a decoder layer's feed-forward part ---------------------------------------------------------

@dataclasses.dataclass
class GatedLayers(_Kept):
    """The two projections of a gated feed-forward part as layers of any kind; two in mixed precision are launched together."""
    gate: Layer
    up: Layer

    def _make(self) -> Optional[B.LutMatvecGroupCall]:
        both = isinstance(self.gate, P.Deployed) and isinstance(self.up, P.Deployed)
        return P.group_products([self.gate, self.up]) if both else None

    def apply(self, X: Inputs, ws: B.Workspace, status: Optional[torch.Tensor] = None, X_up: Optional[Inputs] = None):
        """Both projections of X [m, d_in].  `X_up`: what `up` takes, if that is of another type."""
        if self._args is None:
            inputs = (X, X if X_up is None else X_up)
            return tuple(_as_matrix(apply_layer(l, x, ws, status)) for l, x in zip((self.gate, self.up), inputs))
        X = X.to(torch.float16)
        Y = [torch.empty((X.shape[0], l.d_out), dtype=torch.float32, device=X.device) for l in (self.gate, self.up)]
        if X.shape[0]:
            self._args([X, X], Y, ws)
        return tuple(Y)


def _as_matrix(Y: torch.Tensor) -> torch.Tensor:
    return Y if Y.stride(1) == 1 or Y.shape[1] == 1 else Y.contiguous()


def feed_forward_block(X: torch.Tensor, norm: RmsNorm, gate_up: Union[Int8GatedWeight, GatedLayers], down: Layer,
                       ws: B.Workspace, add: Optional[torch.Tensor] = None, activation: Optional[str] = "silu",
                       status: Optional[torch.Tensor] = None, hidden_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """A decoder layer's gated feed-forward part on the residual stream: s + down(act(gate n) * (up n)), n the norm of s = X
    [rows, hidden] (+ `add`, what the layer's attention gave, in any type).  The projections may be of different kinds, as in
    `attention_block` (all in 8 bits, it is one call); the answer has X's type.  `hidden_dtype`: what `down` is handed, by default X's type, or
    float16 where `down` is in mixed precision, which reads that."""
    gated = isinstance(gate_up, Int8GatedWeight)
    if gated and isinstance(down, Int8Weight):
        Y = torch.empty_like(X)
        B.int8_feed_forward(X, norm.weight, norm.eps, gate_up._args, down._args, Y, ws, add, activation, hidden_dtype, status, True)
        return Y
    if hidden_dtype is None:
        hidden_dtype = torch.float16 if isinstance(down, P.Deployed) else X.dtype
    Ns, stream = _normed(X, norm, (gate_up,) if gated else (gate_up.gate, gate_up.up), status, add)
    if gated:
        H = int8_gated_product(gate_up, Ns[0], ws, activation, out_dtype=hidden_dtype, status=status)
    else:
        G, U = gate_up.apply(Ns[0], ws, status, Ns[1])
        H = epilogue(G, activation=activation, times=U, out_dtype=hidden_dtype)
    if isinstance(down, Int8Weight):
        return int8_product(down, H, ws, out_dtype=X.dtype, status=status, residual=stream)
    return epilogue(_as_matrix(apply_layer(down, H, ws, status)), residual=stream, out_dtype=X.dtype)
