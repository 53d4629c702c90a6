"""CPU pin of the oracle's linear attention in chunks: the token after token form's numbers."""
import numpy as np
import pytest

from oracle import layers_oracle as lo


@pytest.mark.parametrize("chunk", [1, 7, 64])
@pytest.mark.parametrize("ld", [[0.5, -0.003], [-0.2, -40.0], [-1e30, 0.0]])
def test_chunks_are_the_recurrence(chunk, ld):
    rng = np.random.default_rng(chunk)
    cu = [0, 70, 70, 71, 200]
    q, k, v = (rng.standard_normal((200, h, 64)) for h in (4, 2, 2))
    S = rng.standard_normal((5, 2, 64, 64))
    args = (q, k, v, cu, np.asarray(ld), S, [0, 1, -1, 9], [3, 1, 7, 0])
    for a, b in zip(lo.linear_attention_in_chunks(*args, chunk=chunk), lo.linear_attention(*args)):
        np.testing.assert_allclose(a, b, rtol=1e-11, atol=1e-11)
    for a, b in zip(lo.linear_attention_in_chunks(*args[:5], scale=2.0, chunk=chunk), lo.linear_attention(*args[:5], scale=2.0)):
        assert (a is None) == (b is None)
        if a is not None:
            np.testing.assert_allclose(a, b, rtol=1e-11, atol=1e-11)
