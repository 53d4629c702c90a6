"""How far a state of linear attention may be from the 64-bit one, relative to its norm (Frobenius), and three mistakes that must be farther.

The bound, in units of F = 2^-24, half a step of float:
  a token's weight: two exponentials and the scale of the state 2 F each, a quotient, two products and the last scaling F each, rounded up to 12.
    The argument of its exp2 is rounded too: a token of age t / |ld| in its chunk is off by t F more and counts e^-t, so that the mean square
    over the tokens is at most that of t under e^-2t, 1 / 2: 1 (or 31 |ld|, the most that a chunk of 32 has).  Tokens' contributions are
    independent, so that errors of that size in each move the norm by no more.
  what is rounded on the way: three additions a token (a product of matrices adds sixteen tokens up in three parts), each off by at most F
    times the state and by F / sqrt 3 on average, in independent directions: the square root of the tokens that are still in the state.
    A sequence that is cut adds up its pieces with two more roundings each."""
import math

import numpy as np
import torch

F = 2.0 ** -24


def _still_there(n, ld):
    """Tokens (or steps) whose roundings the state still holds."""
    forgets = -math.expm1(2 * ld)
    return n if forgets * n <= 1 else 1 / forgets


def state_norm_bound(ld, n, piece):
    sums = math.sqrt(_still_there(min(n, piece), ld))
    joins = math.sqrt(_still_there(-(-n // piece), ld * piece)) if n > piece else 0.0
    return F * (12 + min(1.0, 31 * abs(ld)) + sums + joins)


def norm_error(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def in_two_parts(x):
    """x as the sum of two bf16 numbers."""
    first = torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().double().numpy()
    return first + torch.from_numpy((x - first).astype(np.float32)).bfloat16().double().numpy()


def state(k, v, ld, start, piece, *, values=lambda x: x, decay=lambda x: x):
    """The state after the tokens, `piece` at a time, in 64 bits; `values` is applied to the decayed values and `decay` to the decay of a piece."""
    S = np.array(start, np.float64)
    for lo in range(0, len(k), piece):
        m = min(piece, len(k) - lo)
        w = np.exp(ld * (m - 1.0 - np.arange(m)))[:, None]
        S = float(decay(math.exp(ld * m))) * S + k[lo:lo + m].T @ values(v[lo:lo + m] * w)
    return S
