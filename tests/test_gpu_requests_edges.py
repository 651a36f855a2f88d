"""Calls at the edges of what the requests' header allows."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from tests.test_gpu_requests import _env, _ints, _matrices, say


@pytest.mark.parametrize("group", [4, (1 << 31) - 1, 1 << 31, (1 << 32) - 3, (1 << 32) - 1])
def test_one_matrix_for_all_units(group):
    """A number of units that share A beyond all there are, up to the largest the call takes, means: one A."""
    import torch
    env = _env("C1")
    units, d1, d2 = 3, 100, 64
    say(f"cpvm_prepare: {units} units, a_group {group}")
    w, a, b = (_ints(x) for x in _matrices(np.random.default_rng(4), units, d1, d2, 5, units, True))
    got = env.rq.cpvm_prepare(units, d1, d2, w, a, b, a_group=group)
    assert torch.equal(got, env.rq.cpvm_prepare(units, d1, d2, w, a, b, a_group=units))
