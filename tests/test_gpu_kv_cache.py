"""The paged cache in 8 bits through the public calls: codes and scales bit for bit after every append."""
import numpy as np
import pytest
import torch

import serving_reference as R

pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _sums(v):
    return [0] + list(np.cumsum(v))


class Both:
    """A cache on the GPU and its plain form, and a table of pages in no order."""

    def __init__(self, S, seqs, pages_each, heads, dim, page, seed=0):
        self.S, self.dim, self.page, self.heads = S, dim, page, heads
        n = seqs * pages_each + 2
        self.cache = S.make_cache(n, heads, dim, page, DEV)
        g = torch.Generator(device=DEV).manual_seed(seed)
        for t in (self.cache.k, self.cache.v):                   # memory that was something else's before
            t.copy_(torch.randint(0, 256, t.shape, generator=g, device=DEV, dtype=torch.uint8))
        for t in (self.cache.k_scale, self.cache.v_scale):
            t.fill_(float("nan"))
        self.order = np.random.default_rng(seed).permutation(n)[: seqs * pages_each].reshape(seqs, pages_each)
        self.table = _i32(self.order.tolist())
        self.k, self.v = R.Pages(n, heads, page, dim), R.Pages(n, heads, page, dim)
        self.held = [0] * seqs

    def append(self, K, V, new, rotation=None, status=None):
        self.S.kv_append(self.cache, K, V, self.table, _i32(self.held), _i32(_sums(new)), rotation, status)
        torch.cuda.synchronize()
        k, v, at = R.as_f32(K), R.as_f32(V), 0
        for i, n in enumerate(new):
            if rotation is not None:
                x = R.turn(k[at:at + n], self.held[i] + np.arange(n), R.as_f32(rotation.cos), R.as_f32(rotation.sin), rotation.interleaved)
            else:
                x = k[at:at + n]
            self.k.append(x, self.order[i], self.held[i])
            self.v.append(v[at:at + n], self.order[i], self.held[i])
            self.held[i] += n
            at += n

    def check(self):
        for codes, scale, keys, want in ((self.cache.k, self.cache.k_scale, True, self.k), (self.cache.v, self.cache.v_scale, False, self.v)):
            got, s = R.page_codes(codes.cpu().numpy(), keys, self.page, self.dim), scale.cpu().numpy()
            for i, n in enumerate(self.held):
                for p in range(-(-n // self.page)):
                    t, at = min(self.page, n - p * self.page), self.order[i, p]
                    assert np.array_equal(s[at], want.scale[at]), (keys, i, p)
                    assert np.array_equal(got[at, :, :t, :self.dim], want.codes[at, :, :t]), (keys, i, p)
                    assert not got[at, :, :t, self.dim:].any()

    def read(self, first, count, dtype):
        return self.S.kv_read(self.cache, self.table, _i32(first), _i32(_sums(count)), sum(count), dtype)

    def values(self, i, first, count, keys):
        c = self.k if keys else self.v
        at = first + np.arange(count)
        p = self.order[i][at // self.page]
        return c.codes[p, :, at % self.page].astype(np.float64) * c.scale[p][..., None].astype(np.float64)


@pytest.mark.parametrize("dim,page,heads,dtype,rot,inter", [
    (128, 64, 3, torch.float16, 128, False), (128, 32, 2, torch.bfloat16, 64, True), (80, 32, 5, torch.float32, 80, False),
    (64, 96, 1, torch.float16, 0, False), (256, 128, 2, torch.bfloat16, 256, True), (96, 64, 2, torch.float16, 48, False),
    (33, 32, 2, torch.float32, 20, True), (1, 32, 4, torch.float16, 0, False), (192, 1024, 1, torch.float32, 192, False),
    (7, 64, 3, torch.bfloat16, 6, False), (224, 32, 2, torch.float16, 32, True), (36, 64, 2, torch.float16, 36, False)])
def test_appends_bit_for_bit(S, dim, page, heads, dtype, rot, inter):
    g = torch.Generator(device=DEV).manual_seed(dim)
    rng = np.random.default_rng(dim)
    seqs = 5
    rounds = [[1, 0, page, page - 1, 2 * page + 3], [1, 1, 1, 1, 1], [page - 2, 5, 0, 2, page], [1, 1, 1, 1, 0]]
    rounds += [rng.integers(0, 4, seqs).tolist() for _ in range(4)] + [[3 * page + 1, 0, 1, 31, 33]]
    most = max(sum(r[i] for r in rounds) for i in range(seqs))
    both = Both(S, seqs, -(-most // page), heads, dim, page, dim)
    rotation = S.make_rotation(most, rot, 500.0, inter, DEV) if rot else None
    for k, new in enumerate(rounds):
        n = sum(new)
        # values that grow and shrink from call to call, so that pages are coded again
        x = torch.randn((n, 2, heads, dim), generator=g, device=DEV) * float(rng.choice([0.01, 1.0, 30.0]))
        x = x.to(dtype)
        both.append(x[:, 0], x[:, 1], new, rotation)
        both.check()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    count = [max(0, h - 3) for h in both.held]
    for out in TYPES:
        K, V = both.read([3] * seqs, count, out)
        torch.cuda.synchronize()
        u = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[out]
        tiny = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}[out]
        for keys, got in ((True, K), (False, V)):
            want = np.concatenate([both.values(i, 3, c, keys) for i, c in enumerate(count)])
            off = np.abs(got.double().cpu().numpy() - want)
            assert (off <= np.abs(want) * (u + 2.0 ** -24) + tiny).all()
    assert status.item() == 0


def test_strided_and_unaligned_rows(S):
    g = torch.Generator(device=DEV).manual_seed(1)
    for dim, dtype, rot in ((64, torch.float16, 64), (80, torch.bfloat16, 0), (33, torch.float32, 32), (128, torch.float16, 96)):
        both = Both(S, 2, 3, 3, dim, 64)
        rotation = S.make_rotation(192, rot, device=DEV) if rot else None
        for new in ([70, 3], [1, 1], [2, 64]):
            n = sum(new)
            # heads outside rows, an odd offset, a gap behind every row
            x = torch.randn((2, 3, n, dim + 5), generator=g, device=DEV).to(dtype)[..., 3:3 + dim]
            both.append(x[0].transpose(0, 1), x[1].transpose(0, 1), new, rotation)
            both.check()
        wide = torch.full((3, 67, dim + 3), 5.0, device=DEV, dtype=torch.float16)
        K, V = wide[..., 1:1 + dim].transpose(0, 1)[:66], torch.empty((66, 3, dim), dtype=torch.float16, device=DEV)
        from paper_2410_13056_amd import binding as B
        B.kv_read(both.cache._view, both.table, _i32([0, 0]), _i32([0, 60, 66]), K, V)
        k2, v2 = both.read([0, 0], [60, 6], torch.float16)
        torch.cuda.synchronize()
        assert torch.equal(K, k2) and torch.equal(V, v2)
        assert (wide[:, 66] == 5).all() and (wide[..., 0] == 5).all() and (wide[..., 1 + dim:] == 5).all()


def test_other_pages_and_later_tokens_stay(S):
    both = Both(S, 3, 4, 2, 96, 64)
    x = torch.randn((80, 2, 2, 96), device=DEV)
    both.append(x[:, 0], x[:, 1], [70, 0, 10])
    before = [t.clone() for t in (both.cache.k, both.cache.v, both.cache.k_scale, both.cache.v_scale)]
    y = torch.randn((5, 2, 2, 96), device=DEV) * 0.01              # too small to change a scale
    both.append(y[:, 0], y[:, 1], [3, 0, 2])
    both.check()
    after = [both.cache.k, both.cache.v, both.cache.k_scale, both.cache.v_scale]
    touched = {int(both.order[0, 1]), int(both.order[2, 0])}
    for b, a in zip(before, after):
        for p in range(a.shape[0]):
            if p not in touched:
                assert torch.equal(a[p].nan_to_num(-7.0) if a.is_floating_point() else a[p],
                                   b[p].nan_to_num(-7.0) if b.is_floating_point() else b[p])
    for b, a, keys in ((before[0], after[0], True), (before[1], after[1], False)):
        for p, lo, hi in ((both.order[0, 1], 6, 9), (both.order[2, 0], 10, 12)):
            x0 = R.page_codes(b.cpu().numpy(), keys, 64, 96)[p]
            x1 = R.page_codes(a.cpu().numpy(), keys, 64, 96)[p]
            assert np.array_equal(x0[:, :lo], x1[:, :lo]) and np.array_equal(x0[:, hi:], x1[:, hi:])


@pytest.mark.parametrize("seqs", [1, 63, 64, 65, 200])
def test_many_sequences_one_token_each_step(S, seqs):
    g = torch.Generator(device=DEV).manual_seed(seqs)
    both = Both(S, seqs, 2, 1, 40, 32)
    first = [(7 * i) % 33 for i in range(seqs)]
    x = torch.randn((sum(first), 2, 1, 40), generator=g, device=DEV).half()
    both.append(x[:, 0], x[:, 1], first)
    for step in range(4):
        x = torch.randn((seqs, 2, 1, 40), generator=g, device=DEV).half() * (step + 1)
        both.append(x[:, 0], x[:, 1], [1] * seqs)
    both.check()


def test_non_finite_values_are_flagged_and_keep_finite_scales(S):
    from paper_2410_13056_amd import binding as B
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    both = Both(S, 2, 2, 2, 48, 32)
    x = torch.randn((20, 2, 2, 48), device=DEV)
    both.append(x[:, 0], x[:, 1], [15, 5], status=status)
    assert status.item() == 0
    x[3, 0, 1, 7], x[4, 1, 0, 0], x[5, 1, 0, 47] = float("nan"), float("inf"), float("-inf")
    both.append(x[:, 0], x[:, 1], [15, 5], status=status)
    both.check()
    assert status.item() == B.STATUS_NONFINITE


def test_values_of_zero_and_of_the_smallest_scale(S):
    both = Both(S, 1, 2, 1, 32, 32)
    x = torch.zeros((5, 2, 1, 32), device=DEV)
    both.append(x[:, 0], x[:, 1], [5])
    both.append(x[:, 0] + 1e-42, x[:, 1] - 1e-40, [5])
    both.append(x[:, 0] + 3e38, x[:, 1], [5])
    both.check()


def test_what_lies_outside_the_tables_is_left_out_and_flagged(S):
    from paper_2410_13056_amd import binding as B
    def run(change, good):
        both = Both(S, 4, 2, 2, 64, 32, seed=9)
        x = torch.randn((12, 2, 2, 64), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2)).half()
        both.append(x[:, 0], x[:, 1], [3, 3, 3, 3])
        table, held, cu = both.table.clone(), [3, 3, 3, 3], [0, 3, 6, 9, 12]
        held, cu = change(table, held, cu)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        S.kv_append(both.cache, x[:, 0], x[:, 1], table, _i32(held), _i32(cu), status=status)
        torch.cuda.synchronize()
        assert status.item() == B.STATUS_RANGE
        both.held = [3] * 4
        for i in good:
            both.k.append(R.as_f32(x[3 * i:3 * i + 3, 0]), both.order[i], 3)
            both.v.append(R.as_f32(x[3 * i:3 * i + 3, 1]), both.order[i], 3)
            both.held[i] = 6
        both.check()
        K, V = S.kv_read(both.cache, table, _i32(held), _i32(cu), 12, torch.float32, status)
        torch.cuda.synchronize()
    def page_out(value):
        def change(table, held, cu):
            table[1, 0] = value
            return held, cu
        return change
    run(page_out(-1), [0, 2, 3])
    run(page_out(10), [0, 2, 3])
    run(page_out(2 ** 31 - 1), [0, 2, 3])
    run(lambda t, h, c: ([3, -2, 3, 3], c), [0, 2, 3])
    run(lambda t, h, c: ([3, 64, 3, 3], c), [0, 2, 3])            # no page for them
    run(lambda t, h, c: ([3, 3, 3, 2 ** 31 - 5], c), [0, 1, 2])
    run(lambda t, h, c: (h, [0, 3, 6, 9, 900]), [0, 1, 2, 3])      # rows beyond the call's
    run(lambda t, h, c: (h, [0, 3, 6, 9, -4]), [0, 1, 2])
    # a sequence that leaves its table in the middle: what fits is written
    both = Both(S, 1, 2, 1, 32, 32, seed=3)
    x = torch.randn((70, 2, 1, 32), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    S.kv_append(both.cache, x[:, 0], x[:, 1], both.table, _i32([0]), _i32([0, 70]), status=status)
    torch.cuda.synchronize()
    assert status.item() == B.STATUS_RANGE
    both.k.append(R.as_f32(x[:64, 0]), both.order[0], 0)
    both.v.append(R.as_f32(x[:64, 1]), both.order[0], 0)
    both.held = [64]
    both.check()


def test_positions_beyond_the_rotation_take_its_last_row(S):
    from paper_2410_13056_amd import binding as B
    both = Both(S, 1, 2, 1, 32, 32)
    rotation = S.make_rotation(20, 32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    x = torch.randn((30, 2, 1, 32), device=DEV)
    both.append(x[:20, 0], x[:20, 1], [20], rotation, status)
    assert status.item() == 0
    both.append(x[20:, 0], x[20:, 1], [10], rotation, status)
    assert status.item() == B.STATUS_RANGE
    both.check()


def test_graph_replays(S):
    both = Both(S, 3, 2, 2, 64, 32)
    x = torch.randn((3, 2, 2, 64), device=DEV).half()
    held, cu = _i32([5, 31, 32]), _i32([0, 1, 2, 3])
    S.kv_append(both.cache, x[:, 0], x[:, 1], both.table, held, cu)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.kv_append(both.cache, x[:, 0], x[:, 1], both.table, held, cu)
    K, V = (torch.empty((3, 2, 64), device=DEV) for _ in range(2))
    from paper_2410_13056_amd import binding as B
    for k in range(3):
        x.copy_(torch.randn((3, 2, 2, 64), device=DEV).half() * (k + 1))
        both.cache.k_scale.zero_(), both.cache.v_scale.zero_()
        graph.replay()
        B.kv_read(both.cache._view, both.table, held, cu, K, V)
        torch.cuda.synchronize()
        step = x.float().abs().amax(-1) / 127
        assert ((K - x[:, 0].float()).abs() <= step[:, 0, :, None] * 0.51).all()
        assert ((V - x[:, 1].float()).abs() <= step[:, 1, :, None] * 0.51).all()


def test_refusals(S):
    cache = S.make_cache(4, 2, 64, 32, DEV)
    K, t, h, cu = torch.randn((3, 2, 64), device=DEV), _i32([[0, 1]]), _i32([0]), _i32([0, 3])
    for bad in (dict(K=K[:, :1]), dict(K=K[..., :63]), dict(K=K[:2]), dict(K=K.half()), dict(V=K.transpose(1, 2)),
                dict(table=t.long()), dict(table=t[0]), dict(held=_i32([0, 0])), dict(cu=_i32([0])), dict(K=K.cpu())):
        a = {"K": K, "V": K, "table": t, "held": h, "cu": cu, **bad}
        with pytest.raises(ValueError):
            S.kv_append(cache, a["K"], a["V"], a["table"], a["held"], a["cu"])
    with pytest.raises(TypeError):
        S.kv_append(cache, K.int(), K.int(), t, h, cu)
    with pytest.raises(ValueError):
        S.make_cache(4, 2, 257, 32, DEV)
    with pytest.raises(ValueError):
        S.make_cache(4, 2, 64, 48, DEV)
    with pytest.raises(ValueError):
        S.KvCache(cache.k, cache.v, cache.k_scale, cache.v_scale, 64, 64)
    with pytest.raises(ValueError):
        S.Rotation(torch.zeros((4, 8), device=DEV), torch.zeros((4, 7), device=DEV))
    from paper_2410_13056_amd import binding as B
    with pytest.raises(B.CmpqError) as e:
        S.kv_append(cache, K, K, t, h, cu, S.make_rotation(8, 66, device=DEV))
    assert e.value.code == -2
    S.kv_append(cache, K[:0], K[:0], t, h, _i32([0, 0]))          # nothing to do
    assert S.kv_read(cache, t, h, _i32([0, 0]), 0)[0].shape == (0, 2, 64)


@pytest.mark.parametrize("dim", [8, 40, 72, 128, 160, 176, 208, 256])
@pytest.mark.parametrize("page", [32, 160, 1024])
def test_blocks_of_32_tokens_that_are_new_as_a_whole_or_in_part(S, dim, page):
    """Appends that begin and end at, before and behind the edges of blocks and pages, with rows that are no numbers."""
    from paper_2410_13056_amd import binding as B
    g = torch.Generator(device=DEV).manual_seed(dim + page)
    rounds = [[page, 33], [31, 1], [1, 62], [64, 97], [page - 1, page + 2]]
    both = Both(S, 2, -(-max(sum(r[i] for r in rounds) for i in range(2)) // page), 2, dim, page, dim)
    rotation = S.make_rotation(4 * page + 300, dim // 16 * 16, device=DEV) if dim >= 16 else None
    for k, new in enumerate(rounds):
        x = torch.randn((sum(new), 2, 2, dim), generator=g, device=DEV) * (1.0 + k % 3)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        both.append(x[:, 0].half(), x[:, 1].half(), new, rotation, status)
        both.check()
        assert int(status) == 0
    bad = torch.randn((40, 2, 2, dim), generator=g, device=DEV).half()
    bad[37, 1, 0, dim // 2], bad[2, 1, 1, 0] = float("nan"), float("-inf")
    both.held = [0, 0]
    both.append(bad[:, 0], bad[:, 1], [39, 1], rotation, status)
    both.check()
    assert int(status) == B.STATUS_NONFINITE
