"""Pins of the oracle of the attention layer's operators: library routines, hand-worked cases, brute force."""
import itertools

import numpy as np
import pytest
import scipy.special
import torch

import oracle
from oracle import attention_oracle as ao


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 2), (6, 1)])
def test_attention_equals_a_library_attention_and_logsumexp(hq, hkv):
    rng = np.random.default_rng(hq)
    lengths, D = [5, 0, 1, 23], 16
    cu = _cu(lengths)
    q, k, v = rng.standard_normal((cu[-1], hq, D)), rng.standard_normal((cu[-1], hkv, D)), rng.standard_normal((cu[-1], hkv, D))
    out, lse, absv, top = ao.causal_attention(q, k, v, cu)
    for r, n in enumerate(lengths):
        if n == 0:
            continue
        t = lambda a: torch.from_numpy(a[cu[r]:cu[r + 1]].transpose(1, 0, 2).copy())
        rep = lambda a: t(a).repeat_interleave(hq // hkv, 0)
        want = torch.nn.functional.scaled_dot_product_attention(t(q), rep(k), rep(v), is_causal=True)
        np.testing.assert_allclose(out[cu[r]:cu[r + 1]], want.numpy().transpose(1, 0, 2), rtol=1e-12, atol=1e-14)
        for h in range(hq):
            for i in range(n):
                x = k[cu[r]:cu[r] + i + 1, h // (hq // hkv)] @ q[cu[r] + i, h] / 4.0
                assert abs(lse[h, cu[r] + i] - scipy.special.logsumexp(x)) < 1e-12
    assert (np.abs(out) <= absv + 1e-12).all() and (top >= 0).all()


def test_attention_by_hand_and_after_earlier_context():
    # logits ln 1, ln 2, ln 3 for the third token: weights 1/6, 2/6, 3/6
    q = np.array([[[1.0]], [[1.0]], [[1.0]]])
    k = np.log(np.array([[[1.0]], [[2.0]], [[3.0]]]))
    v = np.array([[[6.0]], [[12.0]], [[-2.0]]])
    out, lse, _, _ = ao.causal_attention(q, k, v, [0, 3], scale=1.0)
    np.testing.assert_allclose(out[:, 0, 0], [6.0, 10.0, 1 + 4 - 1], rtol=1e-14)
    np.testing.assert_allclose(lse[0], np.log([1.0, 3.0, 6.0]), rtol=1e-14)
    # the last token alone, the others as its context: the same row
    tail = ao.causal_attention(q[2:], k, v, [0, 1], [0, 3], scale=1.0)
    np.testing.assert_allclose(tail[0][0], out[2], rtol=1e-14)
    # the log-sum-exp is the one that the scoring from log-sum-exps takes
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((40, 4, 8)), rng.standard_normal((40, 2, 8))
    lse = ao.causal_attention(q, k, k, [0, 40])[1]
    np.testing.assert_allclose(oracle.importance_scores_from_lse(q, k, lse, [0, 40], [0, 40], n_obs=7),
                               oracle.importance_scores(q, k, [0, 40], n_obs=7), rtol=1e-12)


def test_bf16_neighbours():
    x = np.array([1.0, 1.0 + 2.0 ** -9, -1.0, -1.0 - 2.0 ** -9, 0.0, -3.1e-39], np.float32)
    assert (ao.bf16_floor(x) <= x).all()
    np.testing.assert_array_equal(ao.bf16_floor(x)[:4], [1.0, 1.0, -1.0, -1.0 - 2.0 ** -7])
    y = np.array([1.0, 1.0 + 2.0 ** -40, 0.0, 1e-40])
    up = ao.bf16_ceil_nonneg(y)
    assert (up >= y).all() and up[0] == 1.0 and up[1] == 1.0 + 2.0 ** -7 and up[2] == 0.0


def test_quantisation_by_hand():
    # lowest -2, maximum 13: step 1, codes are the rounded distances (ties to even)
    x = np.zeros((1, 1, 64))
    x[0, 0, :6] = [-2.0, 13.0, -1.5, -0.5, 0.5, 0.4]
    code, lo, step = ao.q4_quantise(x)
    assert lo[0, 0, 0] == -2.0 and step[0, 0, 0] == 1.0
    np.testing.assert_array_equal(code[0, 0, :7], [0, 15, 0, 2, 2, 2, 2])
    np.testing.assert_array_equal(ao.q4_values(code, lo, step)[0, 0, :6], [-2, 13, -2, 0, 0, 0])
    rows = ao.q4_pack(code, lo, step)
    assert rows.shape == (1, 36)
    np.testing.assert_array_equal(rows[0, :3], [0xF0, 0x20, 0x22])       # low half first
    np.testing.assert_array_equal(rows[0, 32:], [0x00, 0xC0, 0x80, 0x3F])  # -2 and 1 in bf16, little-endian
    back = ao.q4_unpack(rows, 1, 64)
    np.testing.assert_array_equal(back[0], code)
    assert back[1][0, 0, 0] == -2.0 and back[2][0, 0, 0] == 1.0
    # equal elements: step 0, code 0, the value itself (rounded down to bf16)
    code, lo, step = ao.q4_quantise(np.full((1, 1, 64), 0.75))
    assert (code == 0).all() and step[0, 0, 0] == 0.0 and (ao.q4_values(code, lo, step) == 0.75).all()


def test_quantisation_is_off_by_at_most_half_a_step():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((50, 3, 128)) * np.exp(3 * rng.standard_normal((50, 3, 1)))).astype(np.float32)
    code, lo, step = ao.q4_quantise(x)
    err = np.abs(ao.q4_values(code, lo, step) - x).reshape(50, 3, 2, 64)
    assert (err <= step[..., None] * 0.5 * (1 + 1e-12)).all()
    assert code.max() == 15 and code.min() == 0
    packed = ao.q4_pack(code, lo, step)
    c2, l2, s2 = ao.q4_unpack(packed, 3, 128)
    np.testing.assert_array_equal(c2, code)
    np.testing.assert_array_equal(l2, lo)
    np.testing.assert_array_equal(s2, step)


def test_decode_over_the_cache_is_the_last_row_of_the_attention():
    rng = np.random.default_rng(2)
    n, hq, hkv, D = 37, 6, 2, 64
    q = rng.standard_normal((1, hq, D))
    rows = [ao.q4_pack(*ao.q4_quantise(rng.standard_normal((n, hkv, D)).astype(np.float32))) for _ in range(2)]
    out, lse, mean, W, _, _, _ = ao.decode_attention_q4(q[0], rows[0], rows[1], hkv)
    K, V = (ao.q4_values(*ao.q4_unpack(x, hkv, D)) for x in rows)
    want, want_lse, _, _ = ao.causal_attention(q, K, V, [0, 1], [0, n])
    np.testing.assert_allclose(out, want[0], rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(lse, want_lse[:, 0], rtol=1e-12)
    assert abs(mean.sum() - 1) < 1e-12 and W.shape == (hq, n)
    # the mean weight is the score that a one-row window gives the tokens
    scores = oracle.importance_scores_with_context(q, K, [0, 1], [0, n], n_obs=1)
    np.testing.assert_allclose(mean[-1:], scores, rtol=1e-12)


@pytest.mark.parametrize("seed", range(4))
def test_eviction_by_brute_force(seed):
    rng = np.random.default_rng(seed)
    n, n_sink, n_recent = 9, 2, 1
    mass = rng.integers(0, 4, n).astype(np.float64)
    for budget in range(n_sink + n_recent, n + 2):
        got = ao.evict_tokens(mass, n, budget, n_sink, n_recent)
        if budget >= n:
            np.testing.assert_array_equal(got, np.arange(n))
            continue
        best = None
        for extra in itertools.combinations(range(n_sink, n - n_recent), budget - n_sink - n_recent):
            key = (-sum(mass[i] for i in extra), extra)
            best = key if best is None or key < best else best
        np.testing.assert_array_equal(got, sorted(list(range(n_sink)) + list(best[1]) + list(range(n - n_recent, n))))


def test_page_rows():
    np.testing.assert_array_equal(ao.page_rows([4, 0, 9], 5, 2), [8, 9, 0, 1, 18])
