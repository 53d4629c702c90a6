"""GPU tests of linear attention at the upper end of float's range: states that the recurrence holds are held by every form.
Tolerances as in tests/test_gpu_layers.py (all of them relative; scaling by powers of two changes no rounding)."""
import numpy as np
import pytest

from test_gpu_attention import BF, F32, _say
from test_gpu_layers import Linear

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (64, F32), (128, F32)])
@pytest.mark.parametrize("lengths,step", [([60, 33], False), ([200, 64], False), ([1, 1], True)])
def test_states_of_2_to_the_110(lengths, step, D, dtype):
    # a chunk at e^-0.5 a token decays by 2^-23; heads that remember more and less beside it
    _say("linear attention, large states", lengths, D, dtype)
    for hq, hkv in ((2, 2), (4, 2)):
        b = Linear(D, lengths, hq, hkv, D, dtype, log_decay=[-0.5, -0.02], starts=[0, -1], stores=[0, 1], step=step)
        b.q *= 2.0 ** -90
        b.k *= 2.0 ** 54
        b.v *= 2.0 ** 53
        b.q64, b.k64, b.v64 = b.q64 * 2.0 ** -90, b.k64 * 2.0 ** 54, b.v64 * 2.0 ** 53
        b.start *= np.float32(2.0 ** 108)
        b.pool *= 2.0 ** 108
        b.run()
        b.check()
        assert 2.0 ** 108 < np.abs(b.results()[1]).max() < 2.0 ** 120
