"""CPU-only tests of the pages behind a drop: the refusals, and the oracle's positions by hand."""
import numpy as np
import pytest

import paper_2605_06221_amd as up
from oracle import layers_oracle as lo

A = 1 << 20            # an aligned address that is never read


def _pages(**kw):
    a = dict(len=A, new=A, dropped=A, seqs=2, page=16, table=A, tstride=8, free=A, num_free=A, left=A, new_len=A, cu=A, cuk=A, pos=A, slots=A, cap=100,
             served=A)
    a.update(kw)
    return up.uniprefill_append_pages_dropped(
        a["len"], a["new"], a["dropped"], a["seqs"], a["page"], a["table"], a["tstride"], a["free"], a["num_free"], a["left"], a["new_len"], a["cu"],
        a["cuk"], a["pos"], a["slots"], a["cap"], a["served"], stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    *[({name: None}, up.UP_ERR_NULL) for name in ("len", "new", "table", "free", "num_free", "left", "new_len", "cu", "cuk", "pos", "slots", "served")],
    *[({name: A + 2}, up.UP_ERR_ALIGN) for name in ("len", "new", "dropped", "table", "free", "num_free", "left", "new_len", "cu", "cuk", "pos", "served")],
    (dict(slots=A + 4), up.UP_ERR_ALIGN), (dict(seqs=-1), up.UP_ERR_SHAPE), (dict(cap=-1), up.UP_ERR_SHAPE), (dict(page=0), up.UP_ERR_RANGE),
    (dict(tstride=-1), up.UP_ERR_RANGE), (dict(cap=2 ** 31 - 2), up.UP_ERR_UNSUPPORTED), (dict(seqs=2 ** 31 - 2), up.UP_ERR_UNSUPPORTED),
    (dict(new_len=A + 4), up.UP_ERR_UNSUPPORTED), (dict(dropped=None, new_len=A - 4), up.UP_ERR_UNSUPPORTED),
])
def test_refusals(kw, want):
    assert _pages(**kw) == want


def test_positions_by_hand():
    table = np.array([[7, 8, -1], [3, -1, -1]])
    got = lo.append_pages([6, 4], [1, 2], 4, table, [20, 21], 2, 5, dropped=[10, -3])
    assert got["pos"] == [16, 4, 5, 0, 0] and got["slots"] == [8 * 4 + 2, 21 * 4, 21 * 4 + 1, -1, -1]
    assert lo.append_pages([6], [3], 4, table, [], 0, 5, dropped=[2 ** 31 - 8])["served"] == 0
    assert lo.append_pages([5], [3], 4, table, [], 0, 3, dropped=[2 ** 31 - 8])["pos"] == [2 ** 31 - 3, 2 ** 31 - 2, 2 ** 31 - 1]
