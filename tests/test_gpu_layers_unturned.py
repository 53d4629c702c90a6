"""GPU test of rotation: elements that do not turn keep their bits, beside whatever they stand."""
import pytest
import torch

from test_gpu_attention import BF, F32, _say
from test_gpu_layers import Rotate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (64, F32), (128, F32)])
@pytest.mark.parametrize("pairs", [False, True])
def test_elements_that_do_not_turn_keep_their_bits(D, dtype, pairs):
    _say("rotate: zeros with signs, largest values and infinities behind the turned part", D, dtype, pairs)
    whole = torch.int32 if dtype == F32 else torch.int16
    for rot in (0, 16, D // 2, D - 16):
        b = Rotate(rot + D, 9, 5, 1, D, dtype, rot=rot, pairs=pairs, norm=False, slots=False)
        rows = b.x.view(9, 7, D)
        odd = torch.tensor([-0.0, 0.0, -1.0, float("inf"), torch.finfo(dtype).max, -0.0, -float("inf"), 3.0], dtype=dtype, device="cuda")
        rows[..., rot:] = odd.repeat((D - rot) // 8)
        rows[..., :rot] = rows[..., :rot].clamp(-3, 3)
        b.run()
        for out, heads in ((b.q_out[:9, :5 * D].view(9, 5, D), rows[:, :5]), (b.k_out[:9, :D].view(9, 1, D), rows[:, 5:6])):
            assert torch.equal(out[..., rot:].contiguous().view(whole), heads[..., rot:].contiguous().view(whole))
            assert torch.isfinite(out[..., :rot]).all()
