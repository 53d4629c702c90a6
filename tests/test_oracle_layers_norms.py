"""CPU tests that the bound on a state's norm is tight enough: what a dropped part of the values, and a decay held in a single float, would do to
the state is beyond it."""
import numpy as np
import pytest

from layers_norms import in_two_parts, norm_error, state, state_norm_bound
from test_oracle_layers import _rng


def _rows(rng, n, d):
    return in_two_parts(rng.standard_normal((n, d))).astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("ld", [-0.05, -0.1, -0.3])
@pytest.mark.parametrize("n", [60, 640])
def test_values_in_two_parts_are_beyond_the_bound(n, ld):
    rng = _rng(n)
    k, v = (_rows(rng, n, 64) for _ in range(2))
    v = np.asarray(in_two_parts(v))
    want = state(k, v, ld, np.zeros((64, 64)), 32)
    assert norm_error(state(k, v, ld, np.zeros((64, 64)), 60), want) < 1e-12
    off = norm_error(state(k, v, ld, np.zeros((64, 64)), 32, values=in_two_parts), want)
    assert off > 1.25 * state_norm_bound(ld, n, 64)


@pytest.mark.parametrize("ld", [-2.107e-05, -3.484e-05])
def test_the_decay_of_a_piece_in_one_float_is_beyond_the_bound(ld):
    rng = _rng(3)
    k, v, start = _rows(rng, 19200, 64), _rows(rng, 19200, 64), 1000 * rng.standard_normal((64, 64))
    want = state(k, v, ld, start, 64)
    off = norm_error(state(k, v, ld, start, 64, decay=np.float32), want)
    assert off > 2 * state_norm_bound(ld, 19200, 64)


@pytest.mark.parametrize("ld", [-2.107e-05, -3.484e-05])
def test_the_decay_of_a_step_in_one_float_is_beyond_the_bound(ld):
    rng = _rng(4)
    k, v, start = _rows(rng, 2000, 64), _rows(rng, 2000, 64), 1000 * rng.standard_normal((64, 64))
    want = state(k, v, ld, start, 1)
    off = norm_error(state(k, v, ld, start, 1, decay=np.float32), want)
    assert off > 2 * state_norm_bound(ld, 2000, 2000)
