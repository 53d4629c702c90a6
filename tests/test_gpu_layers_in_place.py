"""GPU tests of norm and rotation in place: rows that stay where they are, and a single row whatever its strides."""
import pytest
import torch

import paper_2605_06221_amd as up
from test_gpu_attention import _say
from test_gpu_layers import Rotate

pytestmark = pytest.mark.gpu


def test_rows_that_stay_where_they_are():
    _say("rotate: queries, keys and values where they are; queries where they are and the others into slots")
    b = Rotate(1, 77, 8, 2, 128, slots=False)
    b.run()
    b.check()
    c = Rotate(1, 77, 8, 2, 128, slots=False)
    q, k, v = c.views()
    up.uniprefill_norm_rotate(c.p, q, k, v, c.row, c.w[0], c.w[1], c.eps, c.pos, c.freq, c.rot, 0, None, q, c.row, k, c.row, v, c.row, None, 0)
    assert torch.equal(q, b.q_out[:77]) and torch.equal(k, b.k_out[:77]) and torch.equal(v, b.v_out[:77])
    d = Rotate(1, 77, 8, 2, 128)
    q, k, v = d.views()
    up.uniprefill_norm_rotate(d.p, q, k, v, d.row, d.w[0], d.w[1], d.eps, d.pos, d.freq, d.rot, 0, None, q, d.row, d.k_out, d.k_out.shape[1], d.v_out,
                              d.v_out.shape[1], d.slots, d.num)
    d.q_out[:77] = q
    d.check()


def test_a_single_row_in_place_whatever_its_strides():
    _say("rotate: one row in place, another stride")
    b, c = (Rotate(2, 1, 8, 2, 64, slots=False) for _ in range(2))
    b.run()
    q, k, _ = c.views()
    up.uniprefill_norm_rotate(c.p, q, k, None, 0, c.w[0], c.w[1], c.eps, c.pos, c.freq, c.rot, 0, None, q, c.row + 64, k, c.row + 128, None, 0, None, 0)
    assert torch.equal(q, b.q_out[:1]) and torch.equal(k, b.k_out[:1])
