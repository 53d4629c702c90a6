"""GPU tests of the attention layer's operators where lengths, launches and roundings come to their ends."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2605_06221_amd as up
from oracle import attention_oracle as ao
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


def _nearest(x, bits):
    """The number of `bits` significant bits next to the rational x, ties to even (no subnormals)."""
    if x == 0:
        return 0.0
    e = abs(x.numerator).bit_length() - x.denominator.bit_length()
    while abs(x) >= Fraction(2) ** (e + 1):
        e += 1
    while abs(x) < Fraction(2) ** e:
        e -= 1
    return float(round(x / Fraction(2) ** (e - bits + 1)) * Fraction(2) ** (e - bits + 1))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_values_leave_the_cache_rounded_once(dtype):
    """lowest + step * code in rational numbers, rounded to the type, bit for bit: pairs of all distances, whose sums lie next to the
    middle between two bf16 numbers in many places."""
    _say("4-bit load: rounded once", dtype)
    rng = np.random.default_rng(3)
    n, heads, D = 64, 2, 128
    groups = (n, heads, D // 64)
    sig = lambda: 1 + rng.integers(0, 128, groups) / 128.0
    step = sig() * 2.0 ** rng.integers(-3, 4, groups)
    lo = sig() * 2.0 ** rng.integers(-45, 46, groups) * rng.choice([-1, 1], groups)
    step[:4], lo[:4] = 1 + 2.0 ** -7, np.array([-2.0 ** -40, 2.0 ** -40, 0.0, -1.0]).reshape(4, 1, 1)      # 3 * step is a middle
    step[4] = 0.0
    lo[5:8], step[5:8] = -1 - 2.0 ** -7, np.array([2.0 ** -8, 2.0 ** -9, 2.0 ** -30]).reshape(3, 1, 1)
    code = rng.integers(0, 16, (n, heads, D)).astype(np.uint8)
    code[:8, :, 0::16], code[:8, :, 1::16] = 3, 1
    rows = ao.q4_pack(code, lo, step)
    values = [[Fraction(float(lo[i, h, d // 64])) + Fraction(float(step[i, h, d // 64])) * int(code[i, h, d]) for d in range(D)]
              for i in range(n) for h in range(heads)]
    want = torch.tensor([[_nearest(x, 8 if dtype == BF else 24) for x in row] for row in values], dtype=torch.float64).reshape(n, heads, D)
    twice = torch.tensor([[_nearest(Fraction(_nearest(x, 24)), 8) for x in row] for row in values], dtype=torch.float64).reshape(n, heads, D)
    assert dtype == F32 or (twice != want).sum() > 20      # places where a detour over float shows
    out = torch.zeros(n, heads, D, dtype=dtype, device="cuda")
    p = up.make_params(num_seqs=1, total_tokens=1, block_size=64, num_q_heads=heads, num_kv_heads=heads, head_dim=D,
                       qk_dtype=up.UP_F32 if dtype == F32 else up.UP_BF16)
    up.uniprefill_cache_load_q4(p, _dev(rows), None, rows.shape[1], n, _dev(np.arange(n)), n, None, out, None, heads * D)
    torch.cuda.synchronize()
    assert torch.equal(out.double().cpu(), want)


def test_attention_of_very_many_sequences():
    """131072 sequences of one token, 64/64 heads: more work-groups of 512 threads than a launch can count.  A token that sees
    its own key alone has its value, bit for bit, and its logit (a float sum of D products of bf16) as log-sum-exp."""
    n, heads, D = 131072, 64, 64
    _say("attention:", n, "sequences of one token")
    q, k, v = (torch.randn(n, heads, D, dtype=BF, device="cuda") for _ in range(3))
    out = torch.full((n + 1, heads, D), -7.0, dtype=BF, device="cuda")
    lse = torch.full((heads, n), -7.0, device="cuda")
    cu = np.arange(n + 1, dtype=np.int32)
    p = up.make_params(num_seqs=n, total_tokens=n, block_size=64, num_q_heads=heads, num_kv_heads=heads, head_dim=D)
    assert up.uniprefill_attention_plan(p, cu) == (up.UP_OK, 0)
    up.uniprefill_attention(p, q, k, v, heads * D, _dev(cu), cu, None, None, None, 0, 1, out, heads * D, lse, n, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(out[:n], v) and (out[n:] == -7.0).all()
    for lo in range(0, n, 1 << 14):
        a, b = q[lo:lo + (1 << 14)].double(), k[lo:lo + (1 << 14)].double()
        x, size = (a * b).sum(2) / 8, (a * b).abs().sum(2) / 8
        assert ((lse[:, lo:lo + (1 << 14)].double().T - x).abs() <= (D + 4) * F * size + 8 * F * (size + 1)).all()


@pytest.mark.parametrize("lengths,budget,max_len", [
    ([5000, 10, 0, 300, 101, -3], 100, 5000), ([60000, 24577, 0, 9, 8999, 30000, 1 << 30], 9000, 60000), ([7, 0], 10, 0),
])
def test_eviction_updates_lengths_in_place(lengths, budget, max_len):
    """new_len and kv_len_dev at one address: the choice, the rows and the lengths are those of a call with two."""
    _say("eviction: lengths in place", lengths, budget)
    rng = np.random.default_rng(budget)
    R, page, row = len(lengths), 64, 32
    most = min(budget, max_len)
    per, new_per = -(-max_len // page) + 1, -(-most // page) + 1
    table = np.arange(R * per, dtype=np.int32).reshape(R, per)
    new_table = R * per + np.arange(R * new_per, dtype=np.int32).reshape(R, new_per)
    before = _dev(rng.integers(0, 256, (R * (per + new_per) * page, row)).astype(np.uint8))
    mass_host = rng.random((R, max_len + 1)).astype(np.float32)
    mass, tables = _dev(mass_host), (_dev(table), _dev(new_table))
    for _ in range(3):
        found = []
        for in_place in (False, True):
            cache, lens = before.clone(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
            new_len = lens if in_place else torch.full_like(lens, -77)
            kept_idx = torch.full((R, budget), -77, dtype=torch.int32, device="cuda")
            mass_out = torch.full((R, budget), -7.0, device="cuda")
            up.uniprefill_cache_evict(cache, None, row, row, mass, max_len + 1, lens, R, max_len, budget, 4, 6, tables[0], per, tables[1],
                                      new_per, page, kept_idx, mass_out, budget, new_len)
            torch.cuda.synchronize()
            found.append((new_len, cache, kept_idx, mass_out))
        assert found[1][0].tolist() == [min(max(n, 0), max_len, budget) for n in lengths]
        for a, b in zip(*found):
            assert torch.equal(a, b)
    for r, n in enumerate(lengths):
        stay = ao.evict_tokens(mass_host[r], min(max(n, 0), max_len), budget, 4, 6)
        assert found[1][2][r, :len(stay)].tolist() == list(stay) and (found[1][2][r, len(stay):] == -77).all()


@pytest.mark.parametrize("lengths,budget,n_sink,n_recent,page", [
    ([5, 0, 64, 65, 1000], 64, 4, 4, 16), ([3000, 10, 20000], 300, 128, 128, 7), ([60000, 24577, 0, 30000], 9000, 4, 100, 64),
])
def test_eviction_of_one_cache_alone(lengths, budget, n_sink, n_recent, page):
    """v_cache NULL: the keys' rows, indices, masses and lengths as the oracle has them, from a call that nothing came before."""
    _say("eviction of the keys alone", lengths, budget)
    rng = np.random.default_rng(budget + 1)
    R, most, row, stride = len(lengths), max(lengths), 48, 64
    kept = [min(n, budget) for n in lengths]
    old, new = [-(-n // page) for n in lengths], [-(-n // page) for n in kept]
    pages, at = rng.permutation(sum(old) + sum(new)), 0
    table, new_table = np.full((R, max(old)), -1, np.int32), np.full((R, max(new)), -1, np.int32)
    for t, need in ((table, old), (new_table, new)):
        for r, n in enumerate(need):
            t[r, :n] = pages[at:at + n]
            at += n
    before = rng.integers(0, 256, (at * page, stride)).astype(np.uint8)
    mass = rng.integers(0, 200, (R, most)).astype(np.float32)      # ties too
    cache = _dev(before)
    kept_idx, mass_out = torch.full((R, budget), -77, dtype=torch.int32, device="cuda"), torch.full((R, budget), -7.0, device="cuda")
    new_len = torch.full((R,), -77, dtype=torch.int32, device="cuda")
    up.uniprefill_cache_evict(cache, None, row, stride, _dev(mass), most, _dev(np.array(lengths, np.int32)), R, most, budget, n_sink,
                              n_recent, _dev(table), table.shape[1], _dev(new_table), new_table.shape[1], page, kept_idx, mass_out, budget,
                              new_len)
    torch.cuda.synchronize()
    want = before.copy()
    for r, n in enumerate(lengths):
        stay = ao.evict_tokens(mass[r], n, budget, n_sink, n_recent)
        m = len(stay)
        np.testing.assert_array_equal(kept_idx[r, :m].cpu().numpy(), stay)
        np.testing.assert_array_equal(mass_out[r, :m].cpu().numpy(), mass[r][stay])
        assert (kept_idx[r, m:] == -77).all() and (mass_out[r, m:] == -7.0).all()
        want[ao.page_rows(new_table[r], m, page), :row] = before[ao.page_rows(table[r], n, page)[stay], :row]
    assert new_len.tolist() == kept
    np.testing.assert_array_equal(cache.cpu().numpy(), want)
