"""CPU pins of the oracle of the layers between two drops: its functions against other ways to the same numbers."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from oracle import layers_oracle as lo


def _rng(seed):
    return np.random.default_rng(seed)


def test_a_wide_window_is_causal_attention():
    rng = _rng(0)
    cu, ck = np.array([0, 5, 5, 12]), np.array([0, 9, 9, 16])
    q, k, v = rng.standard_normal((12, 4, 64)), rng.standard_normal((16, 2, 64)), rng.standard_normal((16, 2, 64))
    want = ao.causal_attention(q, k, v, cu, ck)
    for window, n_sink in ((9, 0), (1, 9), (5, 4), (10 ** 9, 3)):
        for a, b in zip(lo.window_attention(q, k, v, cu, ck, window, n_sink), want):
            np.testing.assert_allclose(a, b, rtol=1e-13, atol=1e-13)


@pytest.mark.parametrize("window,n_sink", [(1, 0), (3, 0), (2, 4), (7, 1)])
def test_window_attention_against_a_masked_softmax(window, n_sink):
    rng = _rng(window)
    n, m, d = 11, 20, 64
    q, k, v = (torch.from_numpy(rng.standard_normal((x, 1, d))) for x in (n, m, m))
    mask = torch.zeros(n, m, dtype=torch.bool)
    for i in range(n):
        for j in range(m):
            p = m - n + i
            mask[i, j] = j <= p and (p - j < window or j < n_sink)
    want = torch.nn.functional.scaled_dot_product_attention(q[None, :, 0], k[None, :, 0], v[None, :, 0], attn_mask=mask[None])
    got = lo.window_attention(q.numpy(), k.numpy(), v.numpy(), [0, n], [0, m], window, n_sink)
    np.testing.assert_allclose(got[0][:, 0], want[0].numpy(), rtol=1e-12, atol=1e-12)
    if window == 1 and n_sink == 0:
        np.testing.assert_allclose(got[0][:, 0], v[m - n:, 0].numpy())


def test_linear_attention_is_a_sum_over_the_tokens_before():
    rng = _rng(1)
    n, d = 9, 64
    q, k, v = (rng.standard_normal((n, 1, d)) for _ in range(3))
    S0, ld = rng.standard_normal((1, 1, d, d)), np.array([-0.3])
    out, pool, bound, _ = lo.linear_attention(q, k, v, [0, n], ld, S0, [0], [0])
    age = np.arange(n)[:, None] - np.arange(n)
    x = np.where(age >= 0, np.exp(-0.3 * age), 0.0) * (q[:, 0] @ k[:, 0].T)
    want = (x @ v[:, 0] + np.exp(-0.3 * np.arange(1, n + 1))[:, None] * (q[:, 0] @ S0[0, 0])) / 8
    np.testing.assert_allclose(out[:, 0], want, rtol=1e-11, atol=1e-11)
    w = np.exp(-0.3 * np.arange(n - 1, -1, -1))[:, None]
    np.testing.assert_allclose(pool[0, 0], np.exp(-0.3 * n) * S0[0, 0] + (k[:, 0] * w).T @ v[:, 0], rtol=1e-11, atol=1e-11)
    assert (bound >= np.abs(out)).all()
    # in two calls, the second from the first one's state; no decay, and forgetting everything at once
    a = lo.linear_attention(q[:4], k[:4], v[:4], [0, 4], ld, S0, [0], [0])
    b = lo.linear_attention(q[4:], k[4:], v[4:], [0, 5], ld, a[1], [0], [-1])
    np.testing.assert_allclose(np.concatenate([a[0], b[0]]), out, rtol=1e-11, atol=1e-11)
    np.testing.assert_array_equal(b[1], a[1])
    np.testing.assert_allclose(lo.linear_attention(q, k, v, [0, n], [0.5])[0][:, 0], np.tril(q[:, 0] @ k[:, 0].T) @ v[:, 0] / 8, rtol=1e-11, atol=1e-11)
    gone = lo.linear_attention(q, k, v, [0, n], [-np.inf])[0][:, 0]
    np.testing.assert_allclose(gone, (q[:, 0] * k[:, 0]).sum(1)[:, None] * v[:, 0] / 8, rtol=1e-11, atol=1e-11)


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_is_a_complex_product_and_keeps_lengths(pairs):
    rng = _rng(2)
    x, pos, f = rng.standard_normal((5, 3, 64)), np.array([0, 1, 7, 100000, -3]), 10000.0 ** (-np.arange(16) / 16)
    out, size = lo.norm_rotate(x, None, 0.0, pos, f, 32, pairs)
    a, b = (x[..., 0:32:2], x[..., 1:32:2]) if pairs else (x[..., :16], x[..., 16:32])
    z = (a + 1j * b) * np.exp(1j * pos[:, None, None] * f)
    got = (out[..., 0:32:2] + 1j * out[..., 1:32:2]) if pairs else (out[..., :16] + 1j * out[..., 16:32])
    np.testing.assert_allclose(got, z, rtol=1e-9, atol=1e-9)
    np.testing.assert_array_equal(out[..., 32:], x[..., 32:])
    np.testing.assert_array_equal(out[0], x[0])
    assert (size + 1e-12 >= np.abs(out)).all()
    # dot products depend on the distance of two positions alone
    u, w = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    dot = [np.sum(lo.norm_rotate(u, None, 0.0, [p], f, 32, pairs)[0] * lo.norm_rotate(w, None, 0.0, [p + 5], f, 32, pairs)[0]) for p in (0, 900)]
    np.testing.assert_allclose(dot[0], dot[1], rtol=1e-9)
    y = lo.norm_rotate(x, np.full(64, 2.0), 1e-6, pos, f, 32, pairs)[0]
    np.testing.assert_allclose((y * y).mean(-1), 4.0, rtol=1e-4)


def test_pages_by_hand():
    table = np.array([[7, 8, -1], [3, -1, -1], [-1, -1, -1], [5, -1, -1]])
    got = lo.append_pages([6, 4, 0, 1], [1, 1, 5, 0], 4, table, [20, 21, 22, 23], 4, 10)
    assert got["slots"] == [8 * 4 + 2, 23 * 4, 22 * 4, 22 * 4 + 1, 22 * 4 + 2, 22 * 4 + 3, 21 * 4, -1, -1, -1]
    assert got["pos"] == [6, 4, 0, 1, 2, 3, 4, 0, 0, 0]
    assert got["table"].tolist() == [[7, 8, -1], [3, 23, -1], [22, 21, -1], [5, -1, -1]]
    assert (got["new_len"], got["cu"], got["cu_k"], got["served"], got["free_left"]) == ([7, 5, 5, 1], [0, 1, 2, 7, 7], [0, 7, 12, 17, 18], 4, 1)
    # one page short: the third request and all behind it are left
    got = lo.append_pages([6, 4, 0, 1], [1, 1, 5, 1], 4, table, [20, 21], 2, 10)
    assert (got["new_len"], got["served"], got["free_left"], got["cu"]) == ([7, 5, 0, 1], 2, 1, [0, 1, 2, 2, 2])
