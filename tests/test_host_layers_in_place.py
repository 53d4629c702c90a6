"""CPU-only tests of refusals of norm and rotation: an output that starts at its input with another stride, or by slots, is refused before
anything is launched (tests/test_gpu_layers_in_place.py: rows that stay are not), and so is what a launch cannot count."""
import pytest

import paper_2605_06221_amd as up

A, B, C, X, Y, Z = ((i + 1) << 20 for i in range(6))      # aligned addresses that are never read


def _rotate(tokens=100, **kw):
    a = dict(q=A, k=B, v=C, v_stride=2 * 128, q_out=X, qo=8 * 128, k_out=Y, ko=2 * 128, v_out=Z, vo=2 * 128, slots=None)
    a.update(kw)
    p = up.make_params(num_seqs=1, total_tokens=tokens, block_size=64, num_q_heads=8, num_kv_heads=2)
    return up.uniprefill_norm_rotate(p, a["q"], a["k"], a["v"], a["v_stride"], None, None, 1e-6, A, A, 128, 0, None, a["q_out"], a["qo"], a["k_out"],
                                     a["ko"], a["v_out"], a["vo"], a["slots"], 1000, stream=0, check=False)


@pytest.mark.parametrize("kw", [
    dict(q_out=A, qo=9 * 128), dict(k_out=B, ko=3 * 128), dict(v_out=C, vo=3 * 128), dict(v_out=C, v_stride=4 * 128), dict(k_out=B, slots=A),
    dict(v_out=C, slots=A), dict(q=None, q_out=None, k_out=B, slots=A),
])
def test_moving_rows_in_place_is_refused(kw):
    assert _rotate(**kw) == up.UP_ERR_UNSUPPORTED


def test_more_tokens_than_a_launch_has_lanes_for_are_refused():
    assert _rotate(tokens=67108608) == up.UP_ERR_UNSUPPORTED
