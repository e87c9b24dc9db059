"""Serving in 8 bits: what a decoder's attention needs beside the products with the mixed-precision
weights (`pipeline.lut_matvec`, `pipeline.group_products`).

* `prepare_int8`, `int8_product`: a linear layer in 8-bit integers, for layers that are not to go below
  8 bits and for prompts, where multiplications bound the product;
* `KvCache`, `kv_append`, `kv_read`: keys and values in pages of 8-bit codes, keys turned by position on the way in;
* `kv_attention`: attention over the cache, for single tokens, drafts and chunks of prompts;
* `attention_block`: the three together, as a decoder layer's attention runs them.

Everything is enqueued on the current stream and nothing synchronises; there is no gradient, since
codes have none.  `status` ([1] int32, cleared by the caller) collects the flags of `binding.STATUS_*`: codes have no NaN
and no infinity (they become 0 and +-127 codes), so without it such an input goes unnoticed.
"""
from __future__ import annotations

import dataclasses
import functools
from typing import Callable, Optional, Tuple, Union

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


def int8_product(w: Int8Weight, X: torch.Tensor, ws: Optional[B.Workspace] = None,
                 out_dtype: Optional[torch.dtype] = None, out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y [m, d_out] = X [m, d_in] times the weight, X in 8 bits with a scale per token on the way.  `out_dtype`
    defaults to X's."""
    if out is None:
        out = torch.empty((X.shape[0], w.d_out), dtype=out_dtype or X.dtype, device=X.device)
    w._args(X, out, ws or B.Workspace(X.device), status)
    return out


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


def apply_layer(layer: Layer, X: torch.Tensor, ws: B.Workspace, status: Optional[torch.Tensor] = None) -> torch.Tensor:
    """X [m, d_in] times a layer in whichever form it was prepared: 8-bit integers, the mixed-precision tables
    (fp32 out of FP16 in), or any function.  The last two carry a NaN or an infinity on into their outputs; 8-bit
    integers raise it in `status`."""
    if isinstance(layer, Int8Weight):
        return int8_product(layer, X, ws, out_dtype=torch.float32, status=status)
    if isinstance(layer, P.Deployed):
        return P.lut_matvec(layer, X.to(torch.float16), ws)
    return layer(X)


def _as_heads(Y: torch.Tensor, head_dim: int) -> torch.Tensor:
    """[rows, heads * head_dim], of no rows as well, as [rows, heads, head_dim] with unit stride along the dims."""
    Y = Y if Y.stride(1) == 1 else Y.contiguous()
    return Y.reshape(Y.shape[0], Y.shape[1] // head_dim, head_dim)


def attention_block(cache: KvCache, X: torch.Tensor, q: Layer, k: Layer, v: Layer, o: Layer, page_table: torch.Tensor,
                    held: torch.Tensor, lengths: torch.Tensor, cu_rows: torch.Tensor, max_rows: int,
                    max_length: int, ws: B.Workspace, rotation: Optional[Rotation] = None, causal: bool = True,
                    window: int = 0, status: Optional[torch.Tensor] = None,
                    attention_dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """A decoder layer's attention for new tokens X [rows, hidden] of several sequences (see `kv_append`; lengths[i] =
    held[i] + the sequence's rows): the three projections, keys and values into the cache, attention over it, the
    output projection [rows, hidden].  The projections may be of different kinds, for instance queries and outputs in
    mixed precision and the short key and value layers in 8 bits.  `status` collects the flags of all of them.
    `attention_dtype`, float16 or bfloat16: what the attention hands to `o`.  By default bfloat16 for a bfloat16 X, whose
    values may pass float16's range, unless `o` is in mixed precision, which reads float16; else float16."""
    if attention_dtype is None:
        wide = X.dtype == torch.bfloat16 and not isinstance(o, P.Deployed)
        attention_dtype = torch.bfloat16 if wide else torch.float16
    Q, K, V = (_as_heads(apply_layer(layer, X, ws, status), cache.head_dim) for layer in (q, k, v))
    kv_append(cache, K, V, page_table, held, cu_rows, rotation, status)
    O = kv_attention(cache, Q, page_table, lengths, cu_rows, max_rows, max_length, ws, causal=causal, window=window,
                     rotation=rotation, out_dtype=attention_dtype, status=status)
    return apply_layer(o, O.flatten(1), ws, status)
