"""GPU tests of the precision that linear attention's states keep: the difference from the 64-bit state, relative to its norm, within the bound
that tests/layers_norms.py derives (and that tests/test_oracle_layers_norms.py shows to be too small for a dropped part of the values or for a decay
in a single float)."""
import numpy as np
import pytest
import torch

from layers_norms import F, norm_error, state, state_norm_bound
from oracle import layers_oracle as lo
from test_gpu_attention import BF, F32, _rows, _say
from test_gpu_layers import Linear

pytestmark = pytest.mark.gpu


def _check(b, piece, pool, slots):
    """Every head's state of the sequences that store to `slots`, against the oracle's pool."""
    _, got = b.results()
    worst = (0.0,)
    for r, to in enumerate(slots):
        for h in range(b.hkv):
            bound, off = state_norm_bound(float(b.ld[h]), b.lengths[r], piece), norm_error(got[to, h], pool[to, h])
            worst = max(worst, (off / bound, off / F, r, h))
    _say("  worst error / bound, error in 2^-24, sequence, head", *worst)
    assert worst[0] <= 1.0


@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (64, F32), (128, F32)])
@pytest.mark.parametrize("group", [1, 3])
def test_states_of_whole_and_cut_sequences(D, dtype, group):
    _say("linear attention, norms of states", D, dtype, group)
    lengths, slots = [60, 640, 33, 2001], [0, 1, 2, 3]
    b = Linear(D + group, lengths, 3 * group, 3, D, dtype, log_decay=[-0.05, -0.1, -0.3], starts=[-1, -1, -1, -1], stores=slots)
    assert b.ws_bytes == (2 * sum(lengths) // 64 + 1) * 3 * D * D * 4      # (pieces of 64 tokens)
    b.run()
    _check(b, 64, lo.linear_attention_in_chunks(b.q64, b.k64, b.v64, b.cu_host, b.ld, b.start, b.state_in, b.state_out)[1], slots)


@pytest.mark.parametrize("D,dtype,heads", [(64, BF, 32), (128, BF, 32), (256, BF, 16), (64, F32, 32), (128, F32, 16)])
def test_states_of_long_walks(D, dtype, heads):
    _say("linear attention, norms of states, long walks", D, dtype)
    piece = 192
    lengths = [piece, 5 * piece - 7, piece - 1] + [piece - 2] * (13 if heads == 32 else 8)
    slots = list(range(len(lengths)))
    b = Linear(D, lengths, heads, heads, D, dtype, log_decay=-np.geomspace(0.01, 0.4, heads), starts=[-1] * len(lengths), stores=slots)
    assert b.ws_bytes == (2 * sum(lengths) // piece + 1) * heads * D * D * 4 < (2 * sum(lengths) // (piece - 64) + 1) * heads * D * D * 4
    b.run()
    _check(b, piece, lo.linear_attention_in_chunks(b.q64, b.k64, b.v64, b.cu_host, b.ld, b.start, b.state_in, b.state_out)[1], slots)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_long_sequence_decays_by_more_than_a_float(dtype):
    # 300 pieces; the decay of a piece, rounded to one float, would be off by nearly half a step in each
    _say("linear attention, 19200 tokens", dtype)
    b = Linear(4, [19200], 2, 2, 64, dtype, log_decay=[-2.107e-05, -3.484e-05], starts=[0], stores=[0])
    assert b.ws_bytes == (2 * 300 + 1) * 2 * 64 * 64 * 4
    b.start *= np.float32(1000)
    b.pool *= 1000
    b.run()
    _check(b, 64, lo.linear_attention_in_chunks(b.q64, b.k64, b.v64, b.cu_host, b.ld, b.start, b.state_in, b.state_out)[1], [0])


@pytest.mark.parametrize("D,dtype", [(64, BF), (256, BF), (128, F32)])
def test_many_steps_decay_by_more_than_a_float(D, dtype):
    _say("linear attention, 2000 single tokens", D, dtype)
    n = 2000
    rng = np.random.default_rng(D)
    b = Linear(6, [1], 2, 2, D, dtype, log_decay=[-2.107e-05, -3.484e-05], starts=[0], stores=[0], step=True)
    b.start *= np.float32(1000)
    b.pool *= 1000
    (k, k64), (v, v64) = (_rows(rng, dtype, n, 2, D) for _ in range(2))
    k, v = (t.cuda().reshape(n, -1) for t in (k, v))
    for i in range(n):
        b.k[0], b.v[0] = k[i], v[i]
        b.run()
    want = np.zeros((1, 2, D, D))
    for h in range(2):
        want[0, h] = state(k64[:, h], v64[:, h], float(b.ld[h]), b.start[0, h], 100)
    b.lengths = [n]
    _check(b, n, want, [0])
