"""The operators of 8-bit serving, as cases that can be timed and compared.

    product   m tokens times a layer in 8-bit integers, a scale per token and per output channel
    append    keys and values of new tokens, the keys rotated by position, into a paged cache of 8-bit
              codes with a scale per page and head; the pages written are read back as values
    attend    attention of some rows per sequence over such a cache, queries rotated on the way

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` / `run()` do the
work - in plain 32-bit torch, or through the package where `own` is true - and `exact()` says what comes
out by the definition in 64 bits.

A cache holds code + 128 in a byte.  Codes of a page and head lie in pieces of 32 tokens by 32 dims (1 KB), pieces of
the same tokens next to each other; byte [g][t][h][j] of a piece (g < 4, t < 16, h < 2, j < 8) is
    keys     token 16 h + t,                  dim 8 g + j
    values   token 16 (j / 4) + 4 g + j % 4,  dim 16 h + t
and dims beyond the head's are zero codes.
"""
import random

import torch

own = False

DEV = "cuda"
_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"f16": 2, "bf16": 2, "f32": 4}
_TINY = 2.0 ** -126
_BASE = 10000.0


# ---------------------------------------------------------------------------------- cases

def _product(name, m, d_in, d_out, dtype, out):
    return {"name": name, "kind": "product", "m": m, "d_in": d_in, "d_out": d_out, "dtype": dtype, "out": out}


def _append(name, batch, rows, held, kv, dim, page, dtype, rot, inter=False, lens=1):
    """`rows`: most new tokens of a sequence, `held`: most tokens it has before."""
    return {"name": name, "kind": "append", "batch": batch, "rows": rows, "held": held, "kv": kv, "dim": dim,
            "page": page, "dtype": dtype, "rot": rot, "inter": inter, "lens": lens}


def _attend(name, batch, rows, length, kv, group, dim, page, dtype, rot, inter=False, causal=True, window=0,
            mixed=False, empty=False, lens=1):
    """`rows`: most query rows of a sequence, `length`: most tokens it has; `mixed`: every other sequence has one
    row; `empty`: some have no tokens."""
    return {"name": name, "kind": "attend", "batch": batch, "rows": rows, "length": length, "kv": kv, "group": group,
            "dim": dim, "page": page, "dtype": dtype, "rot": rot, "inter": inter, "causal": causal, "window": window,
            "mixed": mixed, "empty": empty, "lens": lens}


def listed():
    return [
        # one token's key projection in the 70B-shaped block: the smallest product, latency counts
        _product("product_1tok_8192x1024", 1, 8192, 1024, "f16", "f32"),
        # sixteen streams through the up projection of a 13B-shaped block: bound by the weight's bytes
        _product("product_16tok_5120x13824", 16, 5120, 13824, "bf16", "bf16"),
        # a short prompt through a layer of sizes that are no multiple of anything (a pruned model)
        _product("product_333tok_4099x3001", 333, 4099, 3001, "f16", "f16"),
        # a prompt of 4096 tokens through the up projection of the 70B-shaped block: the largest
        _product("product_4096tok_8192x28672", 4096, 8192, 28672, "f16", "f16"),
        # a decoding step of 64 sequences, 8 key / value heads of 128 as in the 70B-shaped block
        _append("append_64seq_1tok", 64, 1, 8000, 8, 128, 64, "bf16", 128, lens=5),
        # prompts of a 7B-shaped block (32 heads of 128) entering an empty cache
        _append("append_prompts_6seq", 6, 4000, 0, 32, 128, 64, "f16", 128, lens=6),
        # 80-dim heads, a part of them rotated in interleaved pairs, fp32 straight from a product
        _append("append_chunks_dim80_f32", 9, 300, 700, 12, 80, 32, "f32", 48, True, lens=7),
        # one sequence of a 7B-shaped block, not a page multiple: the smallest, latency counts
        _attend("attend_1seq_777", 1, 1, 777, 32, 1, 128, 64, "f16", 0, lens=8),
        # a decoding step of 64 ragged sequences, 64 query heads on 8
        _attend("attend_64seq_ragged", 64, 1, 8192, 8, 8, 128, 64, "bf16", 128, lens=9),
        # a decoding step of two long documents: few rows, a long axis
        _attend("attend_2seq_131072", 2, 1, 131072, 8, 8, 128, 64, "bf16", 128, lens=10),
        # chunks of three prompts over what is cached of them
        _attend("attend_chunk_3seq", 3, 700, 8000, 8, 8, 128, 64, "f16", 128, lens=11),
        # drafts of up to 6 tokens being checked, 64-dim heads, a sliding window, some sequences new
        _attend("attend_draft_window", 24, 6, 5000, 5, 7, 64, 32, "f16", 64, True, window=1024, empty=True, lens=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["product", "append", "attend"])
    dtype = rng.choice(["f16", "bf16", "f32"])
    if kind == "product":
        m, d_in, d_out = _log_int(rng, 1, 4096), _log_int(rng, 64, 28672), _log_int(rng, 64, 28672)
        while m * d_in * d_out > 4096 * 8192 * 28672:
            m = max(1, m // 2)
        return _without_name(_product("", m, d_in, d_out, dtype, rng.choice(["f16", "bf16", "f32"])))
    kv, dim = rng.choice([1, 2, 4, 5, 8, 12, 16, 32, 40]), rng.choice([32, 64, 80, 96, 128, 128, 192, 256])
    page, inter, lens = rng.choice([32, 64, 128]), rng.random() < 0.3, rng.randrange(1 << 20)
    rot = rng.choice([0, dim, dim, dim // 2])
    if kind == "append":
        batch, rows, held = _log_int(rng, 1, 128), rng.choice([1, _log_int(rng, 2, 8192)]), _log_int(rng, 1, 16384) - 1
        while batch * rows * kv * dim > 6 * 4000 * 32 * 128:
            rows = max(1, rows // 2)
        while batch * (held + rows) * kv * dim > 1 << 30:
            held //= 2
        return _without_name(_append("", batch, rows, held, kv, dim, page, dtype, rot, inter, lens))
    batch, length, rows = _log_int(rng, 1, 128), _log_int(rng, 1, 65536), rng.choice([1, 1, _log_int(rng, 2, 1024)])
    group, dtype = rng.choice([1, 1, 2, 4, 5, 7, 8, 16]), rng.choice(["f16", "bf16"])
    while kv * group > 128:
        group = max(1, group // 2)
    while batch * length * kv * dim > 1 << 28 and length > 64:
        length //= 2
    rows = min(rows, length)
    while batch * rows * length * kv * group > 1 << 30 and rows > 1:
        rows //= 2
    window = _log_int(rng, 16, 4096) if rng.random() < 0.25 else 0
    return _without_name(_attend("", batch, rows, length, kv, group, dim, page, dtype, rot, inter,
                                 rng.random() < 0.85, window, rng.random() < 0.3, rng.random() < 0.2, lens))


def _without_name(case):
    return {k: v for k, v in case.items() if k != "name"}


def _lengths(case):
    """(new rows, tokens held before) or (query rows, tokens) of every sequence: from the case alone."""
    r, n = random.Random(case["lens"]), case["batch"]
    if case["kind"] == "append":
        new = [case["rows"]] + [_log_int(r, 1, case["rows"]) for _ in range(n - 1)]
        return new, [_log_int(r, 1, case["held"] + 1) - 1 for _ in range(n)]
    rows = [case["rows"]] + [_log_int(r, 1, case["rows"]) for _ in range(n - 1)]
    if case["mixed"]:
        rows = [v if i % 2 == 0 else 1 for i, v in enumerate(rows)]
    tokens = [max(q, _log_int(r, max(1, case["length"] // 16), case["length"])) for q in rows]
    tokens[0] = case["length"]
    if case["empty"]:
        tokens = [0 if i % 5 == 4 else t for i, t in enumerate(tokens)]
    return rows, tokens


def _pairs(case):
    """Query-key pairs that the mask leaves, of one head."""
    total = 0
    for q, t in zip(*_lengths(case)):
        for p in range(t - q, t):
            last = p if case["causal"] else t - 1
            first = max(0, p - case["window"] + 1) if case["window"] else 0
            total += max(0, last - first + 1)
    return total


def _reach(case):
    """Tokens whose codes some row of their sequence attends to."""
    total = 0
    for q, t in zip(*_lengths(case)):
        total += t - max(0, t - q - case["window"] + 1) if case["window"] else t
    return total


def work(case):
    if case["kind"] == "product":
        m, i, o = case["m"], case["d_in"], case["d_out"]
        return {"bytes": m * i * _BYTES[case["dtype"]] + i * o + 4 * o + m * o * _BYTES[case["out"]], "flops": 2 * m * i * o}
    es, dim, kv, page = _BYTES[case["dtype"]], case["dim"], case["kv"], case["page"]
    if case["kind"] == "append":
        new, held = _lengths(case)
        values = 2 * sum(new) * kv * dim                               # rows in, codes out
        back = 2 * sum(n + h % page for n, h in zip(new, held)) * kv * dim   # codes in, values out
        return {"bytes": values * (es + 1) + back * (es + 1), "flops": 4 * values + back}
    rows, _ = _lengths(case)
    heads = kv * case["group"]
    return {"bytes": 2 * sum(rows) * heads * dim * es + 2 * _reach(case) * kv * dim, "flops": 4 * heads * dim * _pairs(case)}


# ------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 17)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _dp(case):
    return -(-case["dim"] // 32) * 32


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _sums(counts):
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _tables(case, positions):
    """Cosines and sines of the rotation, [positions, rot / 2]; None where nothing is rotated."""
    if not case["rot"]:
        return None, None
    half = case["rot"] // 2
    freq = torch.pow(_BASE, -torch.arange(half, device=DEV, dtype=torch.float64) / half)
    angle = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * freq
    return angle.cos().float().contiguous(), angle.sin().float().contiguous()


def _pages(case, tokens, g):
    """A table of pages for sequences of so many tokens, in no order, some pages of nobody's."""
    most = max(1, max(-(-t // case["page"]) for t in tokens))
    need = sum(-(-t // case["page"]) for t in tokens)
    total = need + 3
    order = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    counts = [-(-t // case["page"]) for t in tokens]
    table = torch.full((len(tokens), most), -1, dtype=torch.int32)
    at, flat = 0, order.cpu()
    for i, c in enumerate(counts):
        table[i, :c] = flat[at:at + c]
        at += c
    return table.to(DEV), total


def _cache(case, total, g):
    """Codes of normally distributed values, and scales that differ by page and head."""
    size = case["page"] * _dp(case)
    shape = (total, case["kv"], size)
    out = []
    for _ in range(2):
        codes = torch.empty(shape, dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 26) // (case["kv"] * size))
        for a in range(0, total, step):
            b = min(total, a + step)
            codes[a:b] = (_randn(g, b - a, *shape[1:]) * 32).round_().clamp_(-127, 127).add_(128).to(torch.uint8)
        out.append(codes)
    scales = [torch.exp(_randn(g, total, case["kv"]) * 0.3) / 40 for _ in range(2)]
    return {"k": out[0], "v": out[1], "ks": scales[0], "vs": scales[1]}


def prepare(case, seed):
    g = _gen(seed)
    dt = _DTYPE[case["dtype"]]
    if case["kind"] == "product":
        # activations with channels far above the rest, weights with a heavy tail, as real layers have them
        chan = torch.exp(_randn(g, case["d_in"]) * 0.5)
        chan[torch.rand(case["d_in"], generator=g, device=DEV) < 0.005] *= 10
        X = (_randn(g, case["m"], case["d_in"]) * chan).to(dt)
        W = torch.empty((case["d_out"], case["d_in"]), dtype=torch.float16, device=DEV)
        for a in range(0, case["d_out"], 4096):
            w = _randn(g, min(4096, case["d_out"] - a), case["d_in"])
            W[a:a + 4096] = w * 0.02 * (1 + 0.1 * w * w)
        codes, scale = _quantize_rows(W)
        return {"case": case, "X": X, "W": W, "codes": codes, "scale": scale}
    kv, dim, page = case["kv"], case["dim"], case["page"]
    if case["kind"] == "append":
        new, held = _lengths(case)
        total = [n + h for n, h in zip(new, held)]
        table, pages = _pages(case, total, g)
        cos, sin = _tables(case, max(total))
        n = sum(new)
        chan = torch.exp(_randn(g, 2, kv, dim) * 0.4)
        both = (_randn(g, n, 2, kv, dim) * chan).to(dt)             # keys and values of a token next to each other
        first = [h - h % page for h in held]
        back = [t - f for t, f in zip(total, first)]
        return {"case": case, "K": both[:, 0], "V": both[:, 1], "table": table, "held": _ints(held),
                "cu": _ints(_sums(new)), "first": _ints(first), "cu_back": _ints(_sums(back)), "n_back": sum(back),
                "cos": cos, "sin": sin, **_cache(case, pages, g)}
    rows, tokens = _lengths(case)
    table, pages = _pages(case, tokens, g)
    cos, sin = _tables(case, max(max(tokens), 1))
    Q = _randn(g, sum(rows), kv * case["group"], dim).to(dt)
    return {"case": case, "Q": Q, "table": table, "tokens": _ints(tokens), "cu": _ints(_sums(rows)),
            "most_rows": max(rows), "most_tokens": max(tokens), "cos": cos, "sin": sin, **_cache(case, pages, g)}


# -------------------------------------------------------------------------- one pass: own

def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"product": _plain_product, "append": _plain_append, "attend": _plain_attend}[kind](state)
    from paper_2410_13056_amd import binding as B, serving as S
    case = state["case"]
    if "ws" not in state:                       # what a program keeps: its workspace, layer or cache, and rotation
        state["ws"] = B.Workspace(DEV)
        if kind == "product":
            state["layer"] = S.prepare_int8(state["W"])
        else:
            state["cache"] = S.KvCache(state["k"], state["v"], state["ks"], state["vs"], case["page"], case["dim"])
            state["rotation"] = S.Rotation(state["cos"], state["sin"], case["inter"]) if case["rot"] else None
    if kind == "product":
        return S.int8_product(state["layer"], state["X"], state["ws"], out_dtype=_DTYPE[case["out"]])
    if kind == "append":
        S.kv_append(state["cache"], state["K"], state["V"], state["table"], state["held"], state["cu"],
                    rotation=state["rotation"])
        return S.kv_read(state["cache"], state["table"], state["first"], state["cu_back"], state["n_back"],
                         dtype=_DTYPE[case["dtype"]])
    return S.kv_attention(state["cache"], state["Q"], state["table"], state["tokens"], state["cu"],
                          max_rows=state["most_rows"], max_length=state["most_tokens"], ws=state["ws"],
                          causal=case["causal"], window=case["window"], rotation=state["rotation"])


# ------------------------------------------------------------------------ one pass: plain

def _step(most):
    """The scale that gives the largest magnitude the code 127.  Divisions by tensors: torch multiplies by the reciprocal
    of a number instead, which rounds twice."""
    return (most / torch.full_like(most, 127.0)).clamp_min(_TINY)


def _inverse(scale):
    return torch.ones_like(scale) / scale


def _quantize_rows(X):
    """8-bit codes and a scale for each row."""
    x = X.float()
    scale = _step(x.abs().amax(1))
    codes = torch.round(x * _inverse(scale)[:, None]).clamp_(-127, 127).to(torch.int8)
    return codes, scale


def _plain_product(s):
    codes, scale = _quantize_rows(s["X"])
    y = codes.float() @ s["codes"].float().t()
    return (y * scale[:, None] * s["scale"]).to(_DTYPE[s["case"]["out"]])


def _rotate(x, positions, s):
    """x [rows, heads, dim] in 32 bits, turned by the angles of the rows' positions."""
    rot = s["case"]["rot"]
    if not rot:
        return x
    cos, sin = s["cos"][positions][:, None], s["sin"][positions][:, None]
    head, rest = x[..., :rot], x[..., rot:]
    if s["case"]["inter"]:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, rest), -1)


def _rows_of(cu, n):
    """Sequence of each row, and its place in it."""
    seq = torch.searchsorted(cu[1:].contiguous(), torch.arange(n, device=DEV, dtype=torch.int32), right=True)
    return seq, torch.arange(n, device=DEV) - cu[seq].long()


def _spread(codes, keys, case):
    """Stored bytes [..., page * dims] as bytes [..., token, dim]."""
    u, c, lead = case["page"] // 32, _dp(case) // 32, codes.shape[:-1]
    x = codes.view(*lead, u, c, 4, 16, 2, 8)
    n = len(lead)
    if keys:            # u c g t h j -> (u h t) (c g j)
        x = x.permute(*range(n), n, n + 4, n + 3, n + 1, n + 2, n + 5)
    else:               # u c g t h (hi lo) -> (u hi g lo) (c h t)
        x = x.view(*lead, u, c, 4, 16, 2, 2, 4).permute(*range(n), n, n + 5, n + 2, n + 6, n + 1, n + 4, n + 3)
    return x.reshape(*lead, case["page"], _dp(case))


def _gather_in(x, keys, case):
    """The reverse of _spread."""
    u, c, lead = case["page"] // 32, _dp(case) // 32, x.shape[:-2]
    n = len(lead)
    if keys:            # u h t c g j -> u c g t h j
        y = x.view(*lead, u, 2, 16, c, 4, 8).permute(*range(n), n, n + 3, n + 4, n + 2, n + 1, n + 5)
    else:               # u hi g lo c h t -> u c g t h hi lo
        y = x.view(*lead, u, 2, 4, 4, c, 2, 16).permute(*range(n), n, n + 4, n + 2, n + 6, n + 5, n + 1, n + 3)
    return y.reshape(*lead, case["page"] * _dp(case))


def _plain_append(s):
    case, page, dim = s["case"], s["case"]["page"], s["case"]["dim"]
    n = s["K"].shape[0]
    seq, place = _rows_of(s["cu"], n)
    at = s["held"][seq].long() + place                              # position of each new row
    new = s["cu"][1:] - s["cu"][:-1]
    # the pages that get rows: those from the first to the last of each sequence, numbered on
    first = (s["held"] // page).long()
    count = ((s["held"] + new - 1) // page).long() - first + 1
    start = torch.cumsum(count, 0) - count
    touched = start[seq] + at // page - first[seq]
    numbers = torch.arange(int(count.sum()), device=DEV)
    rows = torch.searchsorted(start, numbers, right=True) - 1       # the sequence of each such page
    slot = first[rows] + numbers - start[rows]
    ids = s["table"][rows, slot].long()
    before = (s["held"][rows].long() - slot * page).clamp(0, page)  # tokens that a page has already
    out = []
    for x, codes, scales, keys in ((s["K"], s["k"], s["ks"], True), (s["V"], s["v"], s["vs"], False)):
        x = _rotate(x.float(), at, s) if keys else x.float()
        most = torch.zeros((ids.numel(), case["kv"]), device=DEV)
        most.scatter_reduce_(0, touched[:, None].expand(-1, case["kv"]), x.abs().amax(-1), "amax")
        old = torch.where(before[:, None] > 0, scales[ids], torch.zeros_like(most))
        scale = torch.maximum(old, _step(most))
        inv = _inverse(scale)
        held = _spread(codes[ids], keys, case).float() - 128         # [pages, heads, tokens, dims]
        again = torch.round(held * (old * inv)[:, :, None, None])
        mine = torch.arange(page, device=DEV)[None, :] < before[:, None]
        values = torch.where(mine[:, None, :, None], again, held)
        values[touched, :, at % page, :dim] = torch.round(x * inv[touched][:, :, None]).clamp_(-127, 127)
        values[touched, :, at % page, dim:] = 0
        codes[ids] = _gather_in((values + 128).to(torch.uint8), keys, case)
        scales[ids] = scale
        rseq, rplace = _rows_of(s["cu_back"], s["n_back"])
        pos = s["first"][rseq].long() + rplace
        here = start[rseq] + pos // page - first[rseq]
        out.append((values[here, :, pos % page, :dim] * scale[here][:, :, None]).to(_DTYPE[case["dtype"]]))
    return tuple(out)


def _plain_attend(s):
    case, page, dim = s["case"], s["case"]["page"], s["case"]["dim"]
    kv, group, n = case["kv"], case["group"], s["Q"].shape[0]
    batch, most = s["table"].shape
    seq, place = _rows_of(s["cu"], n)
    rows = (s["cu"][1:] - s["cu"][:-1]).long()
    tokens = s["tokens"].long()
    q = _rotate(s["Q"].float(), (tokens[seq] - rows[seq] + place).clamp(0, max(s["most_tokens"] - 1, 0)), s)
    padded = torch.zeros((batch, s["most_rows"], kv, group, dim), device=DEV)
    padded[seq, place] = q.view(n, kv, group, dim) * dim ** -0.5
    padded = padded.permute(0, 2, 3, 1, 4).reshape(batch, kv, group * s["most_rows"], dim)
    ids = s["table"].long().clamp(0, s["k"].shape[0] - 1)            # [batch, pages]

    def dense(codes, scales, keys):
        x = _spread(codes[ids], keys, case)[..., :dim].float() - 128
        return x * scales[ids][..., None, None]                      # [batch, pages, kv, tokens, dim]

    k = dense(s["k"], s["ks"], True).permute(0, 2, 4, 1, 3).reshape(batch, kv, dim, most * page)
    logits = (padded @ k).view(batch, kv, group, s["most_rows"], most * page)
    del k
    t = torch.arange(most * page, device=DEV)
    p = (tokens - rows)[:, None] + torch.arange(s["most_rows"], device=DEV)        # [batch, rows]
    seen = (t < tokens[:, None, None]).expand(batch, s["most_rows"], most * page)
    if case["causal"]:
        seen = seen & (t <= p[:, :, None])
    if case["window"]:
        seen = seen & (t > p[:, :, None] - case["window"])
    logits = logits.masked_fill_(~seen[:, None, None], float("-inf"))
    top = logits.amax(-1, keepdim=True)
    e = logits.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = e.sum(-1, keepdim=True)
    e = e.div_(torch.where(total == 0, 1.0, total)).view(batch, kv, group * s["most_rows"], most * page)
    v = dense(s["v"], s["vs"], False).permute(0, 2, 1, 3, 4).reshape(batch, kv, most * page, dim)
    o = (e @ v).view(batch, kv, group, s["most_rows"], dim).permute(0, 3, 1, 2, 4)
    return o[seq, place].reshape(n, kv * group, dim).to(_DTYPE[case["dtype"]])


# ---------------------------------------------------------------------------------- exact

def _codes64(x, dims):
    scale = torch.clamp(x.abs().amax(dims, keepdim=True) / 127, min=_TINY)
    return torch.round(x / scale), scale


def _byte_of(case, keys, tokens, dims):
    """Where the byte of a token and dim lies inside a page and head."""
    tokens, dims = tokens[:, None], dims[None, :]
    piece = (tokens // 32) * (_dp(case) // 32) + dims // 32
    t, d = tokens % 32, dims % 32
    if keys:
        return piece * 1024 + (d // 8) * 256 + (t % 16) * 16 + (t // 16) * 8 + d % 8
    return piece * 1024 + (t % 16 // 4) * 256 + (d % 16) * 16 + (d // 16) * 8 + (t // 16) * 4 + t % 4


def _codes_of(s, i, positions, keys):
    """Codes [token, head, dim] of a sequence's positions and their scales [token, head], in 64 bits."""
    case = s["case"]
    ids = s["table"][i].long()[positions // case["page"]]
    byte = _byte_of(case, keys, positions % case["page"], torch.arange(case["dim"], device=DEV))
    codes, scales = (s["k"], s["ks"]) if keys else (s["v"], s["vs"])
    got = codes[ids[:, None, None], torch.arange(case["kv"], device=DEV)[None, :, None], byte[:, None, :]]
    return got.double() - 128, scales[ids].double()


def _turn64(x, positions, s):
    rot, out = s["case"]["rot"], x.clone()
    if rot:
        lanes = torch.arange(rot // 2, device=DEV)
        ia, ib = (2 * lanes, 2 * lanes + 1) if s["case"]["inter"] else (lanes, lanes + rot // 2)
        z = torch.complex(x[..., ia], x[..., ib]) * torch.complex(s["cos"][positions].double(), s["sin"][positions].double())[:, None]
        out[..., ia], out[..., ib] = z.real, z.imag
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "product":
        if case["m"] * case["d_in"] * case["d_out"] > 1 << 41:
            return None
        cx, sx = _codes64(s["X"].double(), 1)
        y = torch.empty((case["m"], case["d_out"]), dtype=torch.float64, device=DEV)
        for a in range(0, case["d_out"], 4096):
            cw, sw = _codes64(s["W"][a:a + 4096].double(), 1)
            y[:, a:a + 4096] = (cx @ cw.t()) * sx * sw.t()
        return y
    if case["kind"] == "append":
        new, held = _lengths(case)
        cu, page, outs = _sums(new), case["page"], ([], [])
        for i in range(len(new)):
            here = torch.arange(held[i], held[i] + new[i], device=DEV)
            k = _turn64(s["K"][cu[i]:cu[i + 1]].double(), here, s)
            v = s["V"][cu[i]:cu[i + 1]].double()
            base = held[i] - held[i] % page
            for x, out, keys in ((k, outs[0], True), (v, outs[1], False)):
                short = held[i] - base                                # tokens of the first page already there
                end = -(-(held[i] + new[i] - base) // page) * page
                full = torch.zeros((end, case["kv"], case["dim"]), dtype=torch.float64, device=DEV)
                full[short:short + new[i]] = x
                old = torch.zeros((1, case["kv"]), dtype=torch.float64, device=DEV)
                if short:
                    codes, scales = _codes_of(s, i, torch.arange(base, held[i], device=DEV), keys)
                    old = scales[:1]
                parts = full.view(-1, page, case["kv"], case["dim"])
                scale = torch.clamp(parts.abs().amax((1, 3)) / 127, min=_TINY)
                scale[0] = torch.maximum(scale[0], old[0])
                got = torch.round(parts / scale[:, None, :, None]) * scale[:, None, :, None]
                got = got.reshape(end, case["kv"], case["dim"])
                if short:
                    got[:short] = torch.round(codes * (old / scale[:1])[:, :, None]) * scale[:1][:, :, None]
                out.append(got[:short + new[i]])
        return tuple(torch.cat(o) for o in outs)
    rows, tokens = _lengths(case)
    if sum(q * t for q, t in zip(rows, tokens)) * case["kv"] * case["group"] * case["dim"] > 1 << 42:
        return None
    cu, out = _sums(rows), []
    for i, (q, t) in enumerate(zip(rows, tokens)):
        o = torch.zeros((q, case["kv"], case["group"], case["dim"]), dtype=torch.float64, device=DEV)
        out.append(o.view(q, -1, case["dim"]))
        if t == 0:
            continue
        p = torch.arange(t - q, t, device=DEV)
        x = _turn64(s["Q"][cu[i]:cu[i + 1]].double(), p.clamp(min=0), s).view(q, case["kv"], case["group"], case["dim"])
        at = torch.arange(t, device=DEV)
        (kc, ks), (vc, vs) = _codes_of(s, i, at, True), _codes_of(s, i, at, False)
        off = torch.zeros((q, t), dtype=torch.float64, device=DEV)
        if case["causal"]:
            off[at[None] > p[:, None]] = float("-inf")
        if case["window"]:
            off[at[None] <= p[:, None] - case["window"]] = float("-inf")
        for h in range(case["kv"]):
            k, v = kc[:, h] * ks[:, h:h + 1], vc[:, h] * vs[:, h:h + 1]
            for a in range(0, q, 128):                                # rows in parts: a long cache times many rows
                w = x[a:a + 128, h].reshape(-1, case["dim"]) @ k.t().contiguous() / case["dim"] ** 0.5
                w = torch.softmax(w + off[a:a + 128].repeat_interleave(case["group"], 0), -1)
                o[a:a + 128, h] = torch.nan_to_num(w @ v).view(-1, case["group"], case["dim"])
    return torch.cat(out)
