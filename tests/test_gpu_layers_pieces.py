"""GPU tests of linear attention where a work-group walks over many chunks: batches whose pieces are several times 64 tokens, against the
64-bit oracle in chunks.  Element by element the tolerances are those of tests/test_gpu_layers.py."""
import numpy as np
import pytest
import torch  # noqa: F401  (before the library, so that both use one HIP runtime)

import paper_2605_06221_amd as up
from oracle import layers_oracle as lo
from test_gpu_attention import BF, F32, _say
from test_gpu_layers import Linear, _slots

pytestmark = pytest.mark.gpu


def _lengths(piece, total):
    """Sequences of pieces and a few tokens more or less, short ones among them, `total` tokens in all."""
    front = [3 * piece + 5, piece, piece - 1, 0, piece + 1, 161, 1, 97, 2 * piece, 33]
    rest = total - sum(front)
    assert rest > 0
    return front + [piece - 40] * (rest // (piece - 40)) + [rest % (piece - 40)]


# type, heads, tokens and the tokens of a piece that follow (tests below assert them)
BATCHES = [
    (64, BF, 32, 32, 4200, 192), (64, BF, 64, 32, 4200, 192), (64, BF, 64, 64, 5100, 448), (128, BF, 32, 32, 4200, 192), (128, BF, 64, 32, 2900, 192),
    (128, BF, 96, 32, 5100, 320), (256, BF, 16, 16, 3000, 192), (256, BF, 32, 16, 3000, 192), (64, F32, 32, 32, 4200, 192), (64, F32, 64, 32, 7000, 320),
    (128, F32, 16, 16, 2900, 192), (128, F32, 32, 16, 2900, 192),
]


@pytest.mark.parametrize("D,dtype,hq,hkv,total,piece", BATCHES)
def test_work_groups_that_walk_over_many_chunks(D, dtype, hq, hkv, total, piece, monkeypatch):
    _say("linear attention, pieces of", piece, D, dtype, hq, hkv)
    monkeypatch.setattr(lo, "linear_attention", lo.linear_attention_in_chunks)
    lengths = _lengths(piece, total)
    starts, stores = _slots(len(lengths))
    # decays that scale the state every chunk, every few and never
    b = Linear(total + D, lengths, hq, hkv, D, dtype, log_decay=-np.geomspace(0.004, 0.8, hkv), starts=starts, stores=stores)
    # (so many bytes and no more: the pieces are as long as that)
    per_add = hkv * D * D * 4
    assert b.ws_bytes == (2 * total // piece + 1) * per_add
    assert b.ws_bytes < (2 * total // (piece - 64) + 1) * per_add
    b.run()
    b.check()


@pytest.mark.parametrize("D,dtype,hq,hkv,piece", [(128, BF, 64, 32, 192), (64, BF, 32, 32, 128)])
def test_whole_sequences_of_many_chunks_beside_none_that_is_cut(D, dtype, hq, hkv, piece, monkeypatch):
    # no workspace: every sequence in one walk, each as long as a piece or nearly
    _say("linear attention, nothing cut", D, dtype)
    monkeypatch.setattr(lo, "linear_attention", lo.linear_attention_in_chunks)
    lengths = [piece, piece - 1, piece - 31, 97, 0, 1] + [piece] * 12
    starts, stores = _slots(len(lengths))
    b = Linear(D, lengths, hq, hkv, D, dtype, log_decay=-np.geomspace(0.004, 0.8, hkv), starts=starts, stores=stores)
    assert b.ws_bytes == 0
    whole = lengths[:-1] + [2 * piece]      # (a longer one is cut: the pieces are about as long as that)
    p = up.make_params(num_seqs=len(whole), total_tokens=sum(whole), block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                       qk_dtype=up.UP_BF16)
    assert up.uniprefill_linear_attention_plan(p, np.concatenate([[0], np.cumsum(whole)]).astype(np.int32))[1] > 0
    b.run()
    b.check()
