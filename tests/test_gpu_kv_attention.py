"""Attention over the paged cache through the public calls, against the softmax in 64 bits over the values that the
codes stand for.

Tolerances.  Roundings on the way: the query (at most 2^-11 of its row's largest magnitude an element), a weight
(2^-11 of itself), the output (2^-11 or 2^-8 of itself) and fp32 arithmetic.  A logit moves by at most `reach` * 2^-11, a
weight's share by a factor of exp(2 * that): an output is off by at most 2 expm1(2 reach 2^-11) + 2^-10 of the largest
value, and its own rounding.  In the 2-norm the four independent contributions stay below 2^-11 each with logits of
order one: 2^-9 in all, and bfloat16 outputs 2^-8 more."""
import numpy as np
import pytest
import torch

import serving_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Setup:
    """A cache of random codes with pages in no order; pages and table entries that belong to nobody hold scales and
    numbers that would show."""

    def __init__(self, S, tokens, heads, dim, page, seed, spread=0.3, size=1 / 40):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.S, self.tokens, self.dim, self.page = S, tokens, dim, page
        counts = [-(-t // page) for t in tokens]
        n = sum(counts) + 3
        self.cache = S.make_cache(n, heads, dim, page, DEV)
        for t in (self.cache.k, self.cache.v):
            t.copy_((torch.randn(t.shape, generator=g, device=DEV) * 32).round().clamp(-127, 127).add(128).to(torch.uint8))
        order = rng.permutation(n)
        most = max(max(counts), 1) + 2
        table = np.full((len(tokens), most), -9, np.int64)
        at = 0
        for i, c in enumerate(counts):
            table[i, :c] = order[at:at + c]
            at += c
        self.table = _i32(table.tolist())
        for t in (self.cache.k_scale, self.cache.v_scale):
            t.copy_(torch.exp(torch.randn(t.shape, generator=g, device=DEV) * spread) * size)
            t[torch.from_numpy(order[at:]).to(DEV)] = float("nan")
        self.order = table

    def dense(self):
        out = []
        for keys, codes, scale in ((True, self.cache.k, self.cache.k_scale), (False, self.cache.v, self.cache.v_scale)):
            x = R.page_codes(codes.cpu().numpy(), keys, self.page, self.dim)[..., :self.dim].astype(np.float64)
            out.append(x * scale.cpu().numpy().astype(np.float64)[:, :, None, None])
        return out

    def want(self, Q, rows, scale, causal, window, rotation):
        q, (k, v), at, out, reach = R.as_f32(Q), self.dense(), 0, [], 0.0
        top = 0.0
        for i, (n, t) in enumerate(zip(rows, self.tokens)):
            x = q[at:at + n]
            if rotation is not None:
                x = R.turn(x, np.maximum(t - n + np.arange(n), 0), R.as_f32(rotation.cos), R.as_f32(rotation.sin), rotation.interleaved)
            ids = self.order[i, :-(-t // self.page)]
            ki, vi = (c[ids].transpose(0, 2, 1, 3).reshape(-1, c.shape[1], self.dim)[:t] for c in (k, v))
            o, r = R.attention(x.astype(np.float64), ki, vi, scale, causal, window)
            out.append(o)
            reach, at = max(reach, r), at + n
            top = max(top, np.abs(vi).max(initial=0.0))
        return np.concatenate(out), reach, top

    def run(self, Q, rows, ws=None, **kw):
        from paper_2410_13056_amd import binding as B
        cu = _i32([0] + list(np.cumsum(rows)))
        return self.S.kv_attention(self.cache, Q, self.table, _i32(self.tokens), cu, max(rows), max(self.tokens),
                                   ws or B.Workspace(DEV), **kw)


def _check(S, setup, rows, heads, dtype, seed=0, causal=True, window=0, rotation=None, scale=None, out=None, q_size=1.0,
           norm=True):
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    Q = (torch.randn((sum(rows), heads, setup.dim), generator=g, device=DEV) * q_size).to(dtype)
    got = setup.run(Q, rows, causal=causal, window=window, rotation=rotation, softmax_scale=scale, out_dtype=out)
    again = setup.run(Q, rows, causal=causal, window=window, rotation=rotation, softmax_scale=scale, out_dtype=out)
    torch.cuda.synchronize()
    assert torch.equal(got, again)
    want, reach, top = setup.want(Q, rows, setup.dim ** -0.5 if scale is None else scale, causal, window, rotation)
    off = np.abs(got.double().cpu().numpy() - want)
    u = 2.0 ** -11 if got.dtype == torch.float16 else 2.0 ** -8
    assert (off <= top * (2 * np.expm1(2 * reach * 2.0 ** -11) + 2.0 ** -10) + u * np.abs(want) + 2.0 ** -24).all(), off.max()
    if norm and np.linalg.norm(want):
        rel = np.linalg.norm(off) / np.linalg.norm(want)
        assert rel <= 2.0 ** -9 + (2.0 ** -8 if got.dtype == torch.bfloat16 else 0), rel
    empty = np.abs(want).sum(-1) == 0
    assert (got.double().cpu().numpy()[empty] == 0).all()
    return got


@pytest.mark.parametrize("dim", [1, 16, 32, 40, 64, 80, 96, 128, 160, 192, 200, 224, 256])
@pytest.mark.parametrize("rows,tokens", [([1, 1, 1], [1, 300, 65]), ([3, 40, 1], [3, 130, 700])])
def test_dims(S, dim, rows, tokens):
    page, dtype = (64, torch.float16) if dim % 3 else (32, torch.bfloat16)
    rot = dim // 2 * 2
    _check(S, Setup(S, tokens, 2, dim, page, dim), rows, 6, dtype, dim,
           rotation=S.make_rotation(max(tokens), rot, 300.0, dim % 64 == 0, DEV) if rot else None)


@pytest.mark.parametrize("group,kv", [(1, 1), (1, 5), (2, 3), (3, 2), (4, 1), (5, 2), (8, 2), (16, 1), (17, 1), (32, 2), (40, 1)])
@pytest.mark.parametrize("most", [1, 2, 5, 19])
def test_groups_of_heads(S, group, kv, most):
    rows = [most, 1, max(1, most - 1), most]
    _check(S, Setup(S, [200, 33, 64, 95], kv, 64, 32, group), rows, group * kv, torch.float16, group)


@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 255, 256, 257, 320, 511, 1025, 5000])
@pytest.mark.parametrize("rows", [1, 4, 70])
def test_lengths(S, tokens, rows):
    _check(S, Setup(S, [tokens, max(1, tokens // 2)], 2, 64, 64, tokens), [min(rows, tokens), 1], 4, torch.float16, tokens)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 7, 32, 100, 4000])
@pytest.mark.parametrize("most", [1, 9, 150])
def test_masks_and_windows(S, causal, window, most):
    rows = [most, min(most, 3), 1, min(most, 40), most]
    tokens = [900, 3, 450, 41, 257 if most < 200 else 300]
    _check(S, Setup(S, tokens, 2, 64, 32, window + most), rows, 6, torch.bfloat16, window, causal, window)


@pytest.mark.parametrize("most", [1, 6, 80])
def test_rows_without_tokens_give_zeros(S, most):
    # sequences without tokens, and with fewer tokens than rows: their first rows see nothing
    rows, tokens = [most, 1, most, most, 2], [0, 0, 77, max(0, most - 3), 1]
    for causal in (True, False):
        for window in (0, 2):
            got = _check(S, Setup(S, tokens, 1, 96, 64, most), rows, 3, torch.float16, most, causal, window)
            assert (got[:rows[0] + 1] == 0).all()


def test_sequences_without_rows(S):
    _check(S, Setup(S, [50, 60, 0, 300], 2, 64, 32, 3), [0, 2, 0, 1], 4, torch.float16)


@pytest.mark.parametrize("seqs", [64, 65, 130])
def test_many_sequences(S, seqs):
    rng = np.random.default_rng(seqs)
    tokens = rng.integers(0, 400, seqs).tolist()
    rows = [int(rng.choice([1, 1, 1, 2, 30])) for _ in range(seqs)]
    _check(S, Setup(S, tokens, 1, 32, 32, seqs), rows, 2, torch.float16, seqs)


@pytest.mark.parametrize("rows", [[1, 1], [3, 1], [200, 1]])
def test_long_sequences_are_cut_and_joined(S, rows):
    _check(S, Setup(S, [20000, 17], 2, 128, 64, 7), rows, 8, torch.bfloat16, 5, rotation=S.make_rotation(20000, 128, device=DEV))


def test_queries_in_32_bits_and_outputs_of_either_type(S):
    s = Setup(S, [130, 40], 2, 80, 32, 2)
    for out in (None, torch.float16, torch.bfloat16):
        got = _check(S, s, [2, 20], 4, torch.float32, out=out, rotation=S.make_rotation(130, 80, device=DEV))
        assert got.dtype == (out or torch.float16)


def test_scales_that_differ_by_many_orders(S):
    # pages from 1e-4 to 1e4 of one another; the norm is that of the largest, so outputs are held to their bound alone
    for seed in range(4):
        s = Setup(S, [640, 100], 2, 64, 32, seed, spread=0.3)
        s.cache.v_scale.mul_(torch.exp(torch.randn(s.cache.v_scale.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)) * 4))
        _check(S, s, [3, 1], 4, torch.bfloat16, seed, norm=False)


def test_values_of_the_smallest_scale_and_of_zero(S):
    s = Setup(S, [200], 1, 64, 32, 3)
    s.cache.v_scale.fill_(2.0 ** -126)
    Q = torch.randn((1, 2, 64), device=DEV).half()
    assert (s.run(Q, [1]) == 0).all()                                # far below FP16
    s = Setup(S, [200], 1, 64, 32, 3)
    first = int(s.order[0, 0])
    s.cache.v_scale[first] = 2.0 ** -126                              # a page of zeros first
    s.cache.v[first] = 128
    _check(S, s, [1], 2, torch.float16)


def test_peaked_and_flat_weights(S):
    s = Setup(S, [1500], 2, 64, 64, 4)
    _check(S, s, [2], 4, torch.float16, scale=2.0, norm=False)        # logits of some tens: a few tokens take all
    _check(S, s, [2], 4, torch.float16, scale=0.0)                    # all alike
    _check(S, s, [2], 4, torch.float16, scale=-0.2)
    _check(S, s, [2], 4, torch.float16, q_size=0.0)
    _check(S, s, [2], 4, torch.float32, q_size=1e-20, scale=1e19)
    _check(S, s, [2], 4, torch.float32, q_size=1e20, scale=1e-21)


def test_one_token_far_above_the_rest(S):
    s = Setup(S, [700], 1, 64, 64, 5)
    s.cache.k.fill_(128)
    page, t = int(s.order[0, 600 // 64]), 600 % 64
    for d in range(64):                                              # token 600 has key (3, 3, ...), the others zero
        piece, x, k = t // 32 * 2 + d // 32, t % 32, d % 32
        s.cache.k[page, 0, piece * 1024 + k // 8 * 256 + x % 16 * 16 + x // 16 * 8 + k % 8] = 255
    s.cache.k_scale.fill_(3.0 / 127)
    Q = torch.full((1, 1, 64), 10.0, device=DEV).half()
    got = s.run(Q, [1])                                              # logit 240 against 0
    v = s.dense()[1][page, 0, t]
    assert np.abs(got[0, 0].double().cpu().numpy() - v).max() <= 2.0 ** -10 * np.abs(v).max()


def test_non_finite_queries_stay_in_their_rows(S):
    s = Setup(S, [300, 90], 2, 64, 32, 6)
    for rows in ([5, 1], [90, 40]):
        Q = torch.randn((sum(rows), 4, 64), device=DEV)
        good = s.run(Q, rows)
        Q[2, 1, 7], Q[4, 3, 0] = float("nan"), float("inf")
        got = s.run(Q, rows)
        bad = torch.zeros((sum(rows), 4), dtype=torch.bool, device=DEV)
        bad[2, 1] = bad[4, 3] = True
        assert torch.equal(got[~bad], good[~bad]) and got[2, 1].isnan().all() and not got[4, 3].isfinite().any()


def test_strides_of_queries_and_outputs(S):
    s = Setup(S, [100, 333], 2, 72, 32, 8)
    for rows in ([1, 1], [20, 61]):
        n = sum(rows)
        base = torch.randn((4, n, 79), device=DEV).half()
        Q = base[..., 3:75].transpose(0, 1)
        whole = torch.full((4, n + 1, 75), 9.0, device=DEV, dtype=torch.float16)
        out = whole[:, :n, 1:73].transpose(0, 1)
        got = s.run(Q, rows, out=out)
        want = s.run(Q.contiguous(), rows)
        assert torch.equal(got, want) and (whole[:, n] == 9).all() and (whole[..., 0] == 9).all() and (whole[..., 73:] == 9).all()


def test_bounds_and_tables_that_do_not_hold_are_flagged(S):
    from paper_2410_13056_amd import binding as B
    s = Setup(S, [100, 200, 64], 1, 64, 32, 9)
    rows, cu = [2, 3, 1], _i32([0, 2, 5, 6])
    Q = torch.randn((6, 2, 64), device=DEV).half()
    good = s.run(Q, rows)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def call(table=s.table, lengths=(100, 200, 64), cu=cu, most=3, length=200, rotation=None):
        status.zero_()
        out = torch.full_like(Q, 5.0)
        S.kv_attention(s.cache, Q, table, _i32(list(lengths)), cu, most, length, B.Workspace(DEV), out=out, status=status,
                       rotation=rotation)
        torch.cuda.synchronize()
        return out, status.item()

    out, st = call()
    assert st == 0 and torch.equal(out, good)
    out, st = call(length=150)                                       # sequence 1 is cut to 150 tokens
    assert st == B.STATUS_RANGE and torch.equal(out[:2], good[:2]) and torch.equal(out[5:], good[5:])
    out, st = call(most=2)                                           # its last row is not done
    assert st == B.STATUS_RANGE and torch.equal(out[:4], good[:4]) and (out[4] == 5).all() and torch.equal(out[5:], good[5:])
    out, st = call(lengths=(100, -4, 64))
    assert st == B.STATUS_RANGE and (out[2:5] == 0).all() and torch.equal(out[:2], good[:2])
    out, st = call(lengths=(2 ** 31 - 1, 200, 64))                   # more than its table has pages for
    assert st == B.STATUS_RANGE and torch.equal(out[2:], good[2:])
    for bad in (-1, s.cache.k.shape[0], 2 ** 31 - 1):                # a page that is none is left out
        table = s.table.clone()
        table[1, 2] = bad
        out, st = call(table=table)
        assert st == B.STATUS_RANGE and torch.equal(out[:2], good[:2]) and torch.equal(out[5:], good[5:])
        k, v = s.dense()
        ids = [p for i, p in enumerate(s.order[1, :7]) if i != 2]
        kk, vv = (c[ids].transpose(0, 2, 1, 3).reshape(-1, 1, 64)[:168] for c in (k, v))
        want, reach = R.attention(R.as_f32(Q[4:5]).astype(np.float64), kk, vv, 64 ** -0.5, True, 0)
        assert np.abs(out[4].double().cpu().numpy() - want[0]).max() <= np.abs(vv).max() * (2 * np.expm1(2 * reach * 2.0 ** -11) + 2.0 ** -9)
    out, st = call(cu=_i32([0, 2, 5, 60]))
    assert st == B.STATUS_RANGE and torch.equal(out[:5], good[:5])
    out, st = call(cu=_i32([0, 2, 5, 1]))
    assert st == B.STATUS_RANGE and torch.equal(out[:5], good[:5]) and (out[5] == 5).all()
    _, st = call(rotation=S.make_rotation(150, 64, device=DEV))
    assert st == B.STATUS_RANGE


def test_another_stream_and_graph_replays(S):
    from paper_2410_13056_amd import binding as B
    for rows, tokens in (([1, 1, 1], [2000, 64, 700]), ([60, 1, 9], [900, 33, 500])):
        s, n = Setup(S, tokens, 2, 64, 32, 12), sum(rows)
        Q, ws = torch.randn((n, 8, 64), device=DEV).half(), B.Workspace(DEV)
        want = s.run(Q, rows, ws).clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = s.run(Q, rows, B.Workspace(DEV))
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        out, cu, lens, graph = torch.empty_like(want), _i32([0] + list(np.cumsum(rows))), _i32(tokens), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            S.kv_attention(s.cache, Q, s.table, lens, cu, max(rows), max(tokens), ws, out=out)
        for k in range(3):                                           # other lengths and queries under the same graph
            lens.copy_(_i32([t - 40 * k if t > 200 else t for t in tokens]))
            Q.copy_(torch.randn((n, 8, 64), device=DEV).half())
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            eager = S.kv_attention(s.cache, Q, s.table, lens, cu, max(rows), max(tokens), B.Workspace(DEV))
            assert torch.equal(out, eager)


def test_cache_beyond_2_to_the_31_bytes(S):
    # the pages of a sequence at the end of a cache whose offsets need more than 32 bits
    heads, dim, page = 8, 128, 64
    n = (1 << 32) // (heads * dim * page) + 40
    cache = S.make_cache(n, heads, dim, page, DEV)
    small = Setup(S, [500], heads, dim, page, 21)
    table = small.table.clone()
    for i, p in enumerate(small.order[0, :8]):
        to = n - 1 - i if i % 2 else i
        for a, b in ((cache.k, small.cache.k), (cache.v, small.cache.v), (cache.k_scale, small.cache.k_scale), (cache.v_scale, small.cache.v_scale)):
            a[to].copy_(b[int(p)])
        table[0, i] = to
    for rows in (1, 50):
        Q, cu, lens = torch.randn((rows, 16, dim), device=DEV).half(), _i32([0, rows]), _i32([500])
        want = S.kv_attention(small.cache, Q, small.table, lens, cu, rows, 500)
        got = S.kv_attention(cache, Q, table, lens, cu, rows, 500)
        assert torch.equal(got, want)
    x = torch.randn((3, 2, heads, dim), device=DEV)
    S.kv_append(cache, x[:, 0], x[:, 1], table, _i32([500]), _i32([0, 3]))
    S.kv_append(small.cache, x[:, 0], x[:, 1], small.table, _i32([500]), _i32([0, 3]))
    a = S.kv_read(cache, table, _i32([490]), _i32([0, 13]), 13)
    b = S.kv_read(small.cache, small.table, _i32([490]), _i32([0, 13]), 13)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals(S):
    from paper_2410_13056_amd import binding as B
    s = Setup(S, [50], 2, 64, 32, 1)
    Q, lens, cu = torch.randn((1, 4, 64), device=DEV).half(), _i32([50]), _i32([0, 1])
    run = lambda **k: S.kv_attention(s.cache, **{"Q": Q, "page_table": s.table, "lengths": lens, "cu_rows": cu, "max_rows": 1, "max_length": 50, **k})
    for bad in (dict(Q=Q[..., :63]), dict(Q=Q[0]), dict(out=torch.empty((2, 4, 64), device=DEV).half()), dict(lengths=lens.long()),
                dict(cu_rows=_i32([0, 1, 1])), dict(page_table=s.table[0]), dict(Q=Q.cpu(), out=Q)):
        with pytest.raises(ValueError):
            run(**bad)
    with pytest.raises(TypeError):
        run(Q=Q.double(), out_dtype=torch.float16)
    for bad in (dict(Q=torch.randn((1, 3, 64), device=DEV)), dict(out_dtype=torch.float32), dict(window=-1), dict(max_rows=-1)):
        with pytest.raises(B.CmpqError) as e:
            run(**bad)
        assert e.value.code == -1
    assert run(Q=Q[:0], cu_rows=_i32([0, 0]), max_rows=0).shape == (0, 4, 64)


def test_attention_block_runs_the_operators_together(S):
    """Mixed kinds of layers, prompt then steps, against the same arithmetic layer by layer."""
    from paper_2410_13056_amd import binding as B
    g = torch.Generator(device=DEV).manual_seed(3)
    hidden, heads, kv, dim, page = 256, 8, 2, 32, 32
    W = {n: torch.randn((o, i), generator=g, device=DEV).half() * i ** -0.5
         for n, o, i in (("q", heads * dim, hidden), ("k", kv * dim, hidden), ("v", kv * dim, hidden), ("o", hidden, heads * dim))}
    layers = {n: S.prepare_int8(w) for n, w in W.items()}
    layers["o"] = lambda x: x.float() @ W["o"].float().t()
    cache, ws, rot = S.make_cache(8, kv, dim, page, DEV), B.Workspace(DEV), S.make_rotation(100, dim, device=DEV)
    table, held = _i32([[5, 1, 0], [2, 7, 3]]), [0, 0]
    for new in ([40, 7], [1, 1], [1, 1], [3, 2]):
        X = torch.randn((sum(new), hidden), generator=g, device=DEV).half()
        lens, cu = [h + n for h, n in zip(held, new)], _i32([0, new[0], sum(new)])
        got = S.attention_block(cache, X, layers["q"], layers["k"], layers["v"], layers["o"], table, _i32(held), _i32(lens),
                                cu, max(new), max(lens), ws, rot)
        q = R.as_f32(S.int8_product(layers["q"], X, ws, out_dtype=torch.float32)).reshape(-1, heads, dim)
        held, parts, at = lens, [], 0
        for i, n in enumerate(new):
            k, v = (t.double().cpu().numpy() for t in S.kv_read(cache, table[i:i + 1].contiguous(), _i32([0]), _i32([0, lens[i]]), lens[i], torch.float32))
            x = R.turn(q[at:at + n], lens[i] - n + np.arange(n), R.as_f32(rot.cos), R.as_f32(rot.sin), False)
            parts.append(R.attention(x.astype(np.float64), k, v, dim ** -0.5, True, 0)[0])
            at += n
        want = np.concatenate(parts).reshape(sum(new), -1) @ W["o"].double().cpu().numpy().T
        rel = np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)
        assert rel <= 2.0 ** -9


class Bounded(Setup):
    """Calls with a bound on the lengths far above them: the work is cut up as for long sequences."""

    def run(self, Q, rows, ws=None, **kw):
        from paper_2410_13056_amd import binding as B
        cu = _i32([0] + list(np.cumsum(rows)))
        return self.S.kv_attention(self.cache, Q, self.table, _i32(self.tokens), cu, max(rows), 1 << 26, ws or B.Workspace(DEV), **kw)


@pytest.mark.parametrize("dim", [1, 32, 40, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("rows,tokens", [([150], [700]), ([3, 90, 1, 17], [3, 130, 700, 65])])
def test_dims_cut_up_as_for_long_sequences(S, dim, rows, tokens):
    _check(S, Bounded(S, tokens, 2, dim, 32, dim + 1), rows, 6, torch.float16, dim,
           rotation=S.make_rotation(max(tokens), dim // 2 * 2, device=DEV) if dim > 1 else None)


@pytest.mark.parametrize("group,kv", [(1, 3), (5, 2), (8, 1), (16, 1), (17, 1), (49, 1)])
def test_groups_cut_up_as_for_long_sequences(S, group, kv):
    _check(S, Bounded(S, [200, 33, 64, 95, 0], kv, 64, 32, group), [77, 1, 2, 60, 3], group * kv, torch.float16, group)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1 << 24])
@pytest.mark.parametrize("tokens", [1, 31, 32, 33, 63, 64, 65, 2049])
def test_lengths_cut_up_as_for_long_sequences(S, causal, window, tokens):
    _check(S, Bounded(S, [tokens, 1, tokens], 2, 128, 64, tokens), [min(100, tokens), 1, 1], 8, torch.bfloat16, causal=causal,
           window=window)


def test_long_sequences_of_many_rows_beside_single_ones(S):
    tokens = [9000, 5, 400, 7000, 33, 2000]
    _check(S, Bounded(S, tokens, 3, 128, 64, 5), [200, 1, 4, 1, 33, 64], 12, torch.bfloat16, 2,
           rotation=S.make_rotation(9000, 128, device=DEV))


def test_many_sequences_cut_up_as_for_long_ones(S):
    rng = np.random.default_rng(8)
    tokens, rows = rng.integers(0, 400, 130).tolist(), [int(rng.choice([0, 1, 1, 2, 70])) for _ in range(130)]
    _check(S, Bounded(S, tokens, 1, 32, 32, 9), rows, 2, torch.float16, 4)
