"""GPU tests of the attention layer's operators where lengths, launches and roundings come to their ends."""
import math

import numpy as np
import pytest
import torch

import paper_2605_06221_amd as up
from test_gpu_attention import BF, F, F32, _dev, _say

pytestmark = pytest.mark.gpu


def test_one_token_after_the_longest_context():
    """2^31 - 65537 keys, the pages of a small cache named over and over: every piece of the cut keys enters the result.
    A query of zeros weighs all keys alike, and column j of every value row is c_j in -2 .. 2, so that sums of a piece
    are whole numbers below 2^24: the output is c_j exactly and the log-sum-exp ln n, up to the float sum of the
    pieces (at most one rounding each), the logarithm's and the product's roundings."""
    n, D, page = (1 << 31) - 65537, 64, 1 << 16
    pages = -(-n // page)
    column = torch.arange(D) % 5 - 2
    k = torch.randn(2 * page, D, device="cuda").to(BF)
    v = column.to(BF).cuda().repeat(2 * page, 1).contiguous()
    table = (torch.arange(pages, dtype=torch.int32, device="cuda") % 2).reshape(1, pages)
    q = torch.zeros(1, D, dtype=BF, device="cuda")
    out, lse = torch.full((1, D), -7.0, dtype=BF, device="cuda"), torch.full((1, 1), -7.0, device="cuda")
    cu, ck = np.array([0, 1], np.int32), np.array([0, n], np.int32)
    p = up.make_params(num_seqs=1, total_tokens=1, block_size=64, num_q_heads=1, num_kv_heads=1, head_dim=D)
    _, ws_bytes = up.uniprefill_attention_plan(p, cu, ck)
    pieces = ws_bytes // (128 * D * 4)      # (about: the float rows of a piece are most of it)
    _say("attention after the longest context:", n, "keys,", pieces, "pieces")
    assert 1 < pieces and n / pieces < 1 << 23      # sums of a piece, at most 2 a key: whole numbers of a float
    ws = torch.empty(ws_bytes + 256, dtype=torch.uint8, device="cuda")
    up.uniprefill_attention(p, q, k, v, D, _dev(cu), cu, _dev(ck), ck, table, pages, page, out, D, lse, 1, ws, ws_bytes)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu()[0], column.to(BF))
    assert abs(float(lse) - math.log(n)) <= pieces * F + 8 * F * math.log(n)
