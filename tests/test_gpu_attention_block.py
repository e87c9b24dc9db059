"""A decoder layer's attention, its operators together: what goes wrong in one shows, whatever kinds the layers are."""
import pytest
import torch

import serving_reference as R  # noqa: F401  (the folder of the tests is on the path)

pytestmark = pytest.mark.gpu

DEV = "cuda"
HIDDEN, HEADS, KV, DIM, PAGE = 256, 8, 2, 32, 32


@pytest.fixture(scope="module")
def S():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2410_13056_amd import binding, serving
    binding.lib()
    return serving


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Block:
    """Layers of either kind, a cache of two sequences; `step` runs the block for new rows of each."""

    def __init__(self, S, kinds="8888", seed=0):
        from paper_2410_13056_amd import binding as B
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.S, self.ws = S, B.Workspace(DEV)
        self.W = {n: torch.randn((o, i), generator=g, device=DEV).half() * i ** -0.5 for n, o, i in
                  (("q", HEADS * DIM, HIDDEN), ("k", KV * DIM, HIDDEN), ("v", KV * DIM, HIDDEN), ("o", HIDDEN, HEADS * DIM))}
        self.layers = {n: S.prepare_int8(w) if kind == "8" else (lambda x, w=w: x.float() @ w.float().t())
                       for (n, w), kind in zip(self.W.items(), kinds)}
        self.cache, self.rot = S.make_cache(8, KV, DIM, PAGE, DEV), S.make_rotation(100, DIM, device=DEV)
        self.table, self.held = _i32([[5, 1, 0], [2, 7, 3]]), [0, 0]
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step(self, X, new, **kw):
        lens, cu = [h + n for h, n in zip(self.held, new)], _i32([0, new[0], sum(new)])
        L = self.layers
        out = self.S.attention_block(self.cache, X, L["q"], L["k"], L["v"], L["o"], self.table, _i32(self.held), _i32(lens), cu,
                                     max(new), max(lens), self.ws, self.rot, status=self.status, **kw)
        torch.cuda.synchronize()
        self.held = lens
        return out


@pytest.mark.parametrize("kinds", ["8888", "8fff", "f8ff", "ff8f", "fff8"])
@pytest.mark.parametrize("new", [[1, 1], [20, 40]])
@pytest.mark.parametrize("value", [float("nan"), float("-inf")])
def test_inputs_that_are_no_finite_numbers_are_flagged(S, kinds, new, value):
    from paper_2410_13056_amd import binding as B
    b = Block(S, kinds)
    X = torch.randn((sum(new), HIDDEN), device=DEV).half()
    b.step(X, new)
    assert b.status.item() == 0
    X[0, 3] = value
    b.step(X[:2], [1, 1])
    assert b.status.item() == B.STATUS_NONFINITE
