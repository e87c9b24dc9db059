"""Activations of strongly negative values in fp32: as long as the value is one, relative to it."""
import numpy as np
import pytest
import torch

import feed_forward_reference as Q
from test_gpu_epilogue import DEV, S  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,low,high", [("silu", -110, -60), ("gelu_tanh", -13, -8)])
def test_tails(S, name, low, high):  # noqa: F811
    """The relative bound of `feed_forward_reference.act`, and half a step of the smallest numbers (rounded up to one): the
    quotient is scaled by a power of two, which is exact but there."""
    v = torch.linspace(low, high, 20001, dtype=torch.float64).float()
    want, rel = Q.act(v.double().numpy(), name)
    got = S.epilogue(v.to(DEV)[None], activation=name)[0].double().cpu().numpy()
    assert (np.abs(got - want) <= rel * np.abs(want) + 2.0 ** -149).all()
    assert (np.abs(want) < 2.0 ** -126).any() and ((got != 0) | (np.abs(want) < 2.0 ** -148)).all()


def test_a_factor_brings_them_back(S):  # noqa: F811
    v = torch.linspace(-95, -80, 3001, dtype=torch.float64).float().to(DEV)[None]
    u = torch.full_like(v, 1e37)
    got = S.epilogue(v, activation="silu", times=u)[0].double().cpu().numpy()
    h, rel = Q.act(Q.f64(v)[0], "silu")
    want = h * float(u[0, 0])
    assert (np.abs(got - want) <= (rel + 2 * Q.HALF) * np.abs(want) + 2.0 ** -149 * float(u[0, 0])).all()
