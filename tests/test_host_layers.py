"""CPU-only tests of the boundary of the operators between two drops: every refusal comes back on the host before anything is
launched (there is no GPU in the process), plans are pure, and empty batches are legal."""
import numpy as np
import pytest

import paper_2605_06221_amd as up

A = 1 << 20            # a 16- and 256-byte aligned address that is never read
CU = np.array([0, 60, 100], np.int32)
CK = np.array([0, 100, 200], np.int32)
NAN, INF = float("nan"), float("inf")
BAD_PARAMETERS = [
    (dict(head_dim=96), up.UP_ERR_UNSUPPORTED), (dict(num_q_heads=9), up.UP_ERR_UNSUPPORTED), (dict(num_q_heads=130), up.UP_ERR_UNSUPPORTED),
    (dict(qk_dtype=3), up.UP_ERR_UNSUPPORTED), (dict(head_dim=256, qk_dtype=up.UP_F32), up.UP_ERR_UNSUPPORTED),
    (dict(softmax_scale=-1.0), up.UP_ERR_RANGE), (dict(softmax_scale=NAN), up.UP_ERR_RANGE), (dict(q_row_stride=100), up.UP_ERR_SHAPE),
    (dict(k_row_stride=2 * 128 + 4), up.UP_ERR_ALIGN), (dict(num_seqs=-1), up.UP_ERR_SHAPE),
]


def _params(**kw):
    base = dict(num_seqs=2, total_tokens=100, block_size=64, num_q_heads=8, num_kv_heads=2)
    base.update(kw)
    return up.make_params(**base)


def _window(p=None, **kw):
    a = dict(q=A, k=A, v=A, v_stride=2 * 128, cu=A, cu_host=CU, cuk=None, cuk_host=None, table=None, tstride=0, page=16, window=10, n_sink=4,
             out=A, out_stride=8 * 128, lse=A, lse_stride=100, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return up.uniprefill_attention_window(p or _params(), a["q"], a["k"], a["v"], a["v_stride"], a["cu"], a["cu_host"], a["cuk"],
                                          a["cuk_host"], a["table"], a["tstride"], a["page"], a["window"], a["n_sink"], a["out"],
                                          a["out_stride"], a["lse"], a["lse_stride"], a["ws"], a["ws_bytes"], stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(window=0), up.UP_ERR_RANGE), (dict(window=-5), up.UP_ERR_RANGE), (dict(n_sink=-1), up.UP_ERR_RANGE),
    (dict(q=None), up.UP_ERR_NULL), (dict(v=None), up.UP_ERR_NULL), (dict(out=None), up.UP_ERR_NULL), (dict(cu=None), up.UP_ERR_NULL),
    (dict(cu_host=None), up.UP_ERR_NULL), (dict(cuk=A), up.UP_ERR_NULL), (dict(table=A, tstride=99), up.UP_ERR_NULL),
    (dict(cu_host=np.array([0, 60, 99], np.int32)), up.UP_ERR_SHAPE),
    (dict(cuk=A, cuk_host=np.array([0, 59, 200], np.int32)), up.UP_ERR_SHAPE), (dict(cuk=A, cuk_host=CK, table=A, tstride=6), up.UP_ERR_SHAPE),
    (dict(cuk=A, cuk_host=CK, table=A, tstride=7, page=0), up.UP_ERR_RANGE), (dict(v_stride=2 * 128 - 8), up.UP_ERR_SHAPE),
    (dict(out_stride=8 * 128 + 4), up.UP_ERR_ALIGN), (dict(lse_stride=99), up.UP_ERR_SHAPE), (dict(lse=A + 2), up.UP_ERR_ALIGN),
    (dict(q=A + 8), up.UP_ERR_ALIGN), (dict(out=A + 8), up.UP_ERR_ALIGN),
])
def test_window_refusals(kw, want):
    assert _window(**kw) == want


@pytest.mark.parametrize("kw,want", BAD_PARAMETERS)
def test_bad_parameters_are_refused(kw, want):
    p = _params(**kw)
    assert _window(p) == want and _linear(p) == want and _rotate(p) == want
    assert up.uniprefill_attention_window_plan(p, CU, None, 10, 4, check=False)[0] == want
    assert up.uniprefill_linear_attention_plan(p, CU, check=False)[0] == want
    s = _params(total_tokens=2, **kw)
    assert _step(s) == want and _state(s) == want and up.uniprefill_attention_window_step_plan(s, 100, 10, 4, check=False)[0] == want


def test_window_plans():
    # one token on a long cache: a wide window is cut, a narrow one is not, and the workspace is asked for
    p = _params(num_seqs=1, total_tokens=1)
    cu, ck = np.array([0, 1], np.int32), np.array([0, 200000], np.int32)
    need = up.uniprefill_attention_window_plan(p, cu, ck, 150000, 4)[1]
    assert need > 0 and need % 256 == 0
    assert up.uniprefill_attention_window_plan(p, cu, ck, 500, 4)[1] == 0
    # (no cut is made that the narrow window does not reach, whatever the numbers)
    for window in (1, 2, 100, 1 << 20, 2 ** 31 - 1):
        for n_sink in (0, 1, 128, 2 ** 31 - 1):
            assert 0 <= up.uniprefill_attention_window_plan(p, cu, ck, window, n_sink)[1] <= up.uniprefill_attention_plan(p, cu, ck)[1] * 2
            assert up.uniprefill_attention_window_step_plan(p, 131072, window, n_sink)[0] == up.UP_OK
    kw = dict(cu_host=cu, cuk=A, cuk_host=ck, window=150000)
    assert _window(p, ws=None, **kw) == up.UP_ERR_WORKSPACE
    assert _window(p, ws_bytes=need - 1, **kw) == up.UP_ERR_WORKSPACE
    assert _window(p, ws=A + 16, **kw) == up.UP_ERR_ALIGN
    assert up.uniprefill_attention_window_plan(p, cu, ck, 0, 4, check=False)[0] == up.UP_ERR_RANGE
    # a long prompt needs none
    p = _params(num_seqs=1, total_tokens=131072, num_q_heads=32, num_kv_heads=8)
    assert up.uniprefill_attention_window_plan(p, np.array([0, 131072], np.int32), None, 4096, 128)[1] == 0


def test_nothing_to_do():
    for lengths in ([], [0, 0, 0]):
        cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        p = _params(num_seqs=len(lengths), total_tokens=0)
        assert _window(p, q=None, k=None, v=None, out=None, lse=None, ws=None, ws_bytes=0, cu_host=cu) == up.UP_OK
        assert _rotate(p, q=None, k=None, q_out=None, k_out=None, v=None, v_out=None, pos=None) == up.UP_OK
    p = _params(num_seqs=0, total_tokens=0)
    assert _step(p, q=None, out=None, kc=None, vc=None, len=None, table=None) == up.UP_OK
    assert _linear(p, q=None, k=None, v=None, out=None, cu_host=np.zeros(1, np.int32)) == up.UP_OK
    assert _state(p, q=None, k=None, v=None, out=None) == up.UP_OK


def _step(p=None, **kw):
    a = dict(q=A, kc=A, vc=A, v_stride=2 * 128, len=A, max_len=100, table=A, tstride=7, page=16, window=10, n_sink=4, out=A, out_stride=8 * 128,
             lse=A, lse_stride=2, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return up.uniprefill_attention_window_step(p or _params(total_tokens=2), a["q"], a["kc"], a["vc"], a["v_stride"], a["len"], a["max_len"],
                                               a["table"], a["tstride"], a["page"], a["window"], a["n_sink"], a["out"], a["out_stride"],
                                               a["lse"], a["lse_stride"], a["ws"], a["ws_bytes"], stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), up.UP_ERR_NULL), (dict(kc=None), up.UP_ERR_NULL), (dict(vc=None), up.UP_ERR_NULL), (dict(len=None), up.UP_ERR_NULL),
    (dict(out=None), up.UP_ERR_NULL), (dict(table=None), up.UP_ERR_NULL), (dict(max_len=-1), up.UP_ERR_SHAPE), (dict(tstride=6), up.UP_ERR_SHAPE),
    (dict(page=0), up.UP_ERR_RANGE), (dict(tstride=-1), up.UP_ERR_RANGE), (dict(window=0), up.UP_ERR_RANGE), (dict(n_sink=-1), up.UP_ERR_RANGE),
    (dict(v_stride=255), up.UP_ERR_SHAPE), (dict(v_stride=260), up.UP_ERR_ALIGN), (dict(out_stride=1000), up.UP_ERR_SHAPE),
    (dict(lse_stride=1), up.UP_ERR_SHAPE), (dict(q=A + 8), up.UP_ERR_ALIGN), (dict(len=A + 2), up.UP_ERR_ALIGN), (dict(table=A + 2), up.UP_ERR_ALIGN),
    (dict(max_len=2 ** 31 - 1, tstride=1 << 40), up.UP_ERR_UNSUPPORTED), (dict(v_stride=1 << 27), up.UP_ERR_UNSUPPORTED),
    (dict(max_len=100000, tstride=1 << 40, window=90000, ws=None), up.UP_ERR_WORKSPACE),
    (dict(max_len=100000, tstride=1 << 40, window=90000, ws=A + 16), up.UP_ERR_ALIGN),
    (dict(max_len=100000, tstride=1 << 40, window=90000, ws_bytes=16), up.UP_ERR_WORKSPACE),
])
def test_step_refusals(kw, want):
    assert _step(**kw) == want
    assert _step(_params()) == up.UP_ERR_SHAPE      # not one token per sequence
    assert up.uniprefill_attention_window_step_plan(_params(), 100, 10, 4, check=False)[0] == up.UP_ERR_SHAPE


LINEAR = dict(q=A, k=A, v=A, v_stride=2 * 128, cu=A, cu_host=CU, decay=A, states=A, state_stride=2 * 128 * 128, num=7, state_in=A, state_out=A,
              out=A, out_stride=8 * 128, ws=A, ws_bytes=1 << 40)


def _linear(p=None, **kw):
    a = dict(LINEAR, **kw)
    return up.uniprefill_linear_attention(p or _params(), a["q"], a["k"], a["v"], a["v_stride"], a["cu"], a["cu_host"], a["decay"], a["states"],
                                          a["state_stride"], a["num"], a["state_in"], a["state_out"], a["out"], a["out_stride"], a["ws"],
                                          a["ws_bytes"], stream=0, check=False)


def _state(p=None, **kw):
    a = dict(LINEAR, **kw)
    return up.uniprefill_linear_attention_step(p or _params(total_tokens=2), a["q"], a["k"], a["v"], a["v_stride"], a["decay"], a["states"],
                                               a["state_stride"], a["num"], a["state_in"], a["state_out"], a["out"], a["out_stride"],
                                               stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), up.UP_ERR_NULL), (dict(k=None), up.UP_ERR_NULL), (dict(v=None), up.UP_ERR_NULL), (dict(out=None), up.UP_ERR_NULL),
    (dict(decay=None), up.UP_ERR_NULL), (dict(states=None), up.UP_ERR_NULL), (dict(states=None, state_in=None), up.UP_ERR_NULL),
    (dict(num=-1), up.UP_ERR_SHAPE), (dict(state_stride=2 * 128 * 128 - 4), up.UP_ERR_SHAPE), (dict(state_stride=2 * 128 * 128 + 2), up.UP_ERR_ALIGN),
    (dict(state_stride=1 << 60), up.UP_ERR_UNSUPPORTED), (dict(v_stride=255), up.UP_ERR_SHAPE), (dict(v_stride=260), up.UP_ERR_ALIGN),
    (dict(out_stride=1000), up.UP_ERR_SHAPE), (dict(states=A + 8), up.UP_ERR_ALIGN), (dict(q=A + 8), up.UP_ERR_ALIGN), (dict(decay=A + 2), up.UP_ERR_ALIGN),
    (dict(state_in=A + 2), up.UP_ERR_ALIGN), (dict(state_out=A + 1), up.UP_ERR_ALIGN),
])
def test_linear_refusals(kw, want):
    assert _linear(**kw) == want and _state(**kw) == want
    assert _linear(cu=None) == up.UP_ERR_NULL and _linear(cu_host=None) == up.UP_ERR_NULL
    assert _linear(cu_host=np.array([0, 60, 99], np.int32)) == up.UP_ERR_SHAPE
    assert _state(_params()) == up.UP_ERR_SHAPE
    cu = np.array([0, 2 ** 30 + 1], np.int32)
    assert up.uniprefill_linear_attention_plan(_params(num_seqs=1, total_tokens=2 ** 30 + 1), cu, check=False)[0] == up.UP_ERR_UNSUPPORTED
    n = 1 << 23
    assert _state(_params(num_seqs=n, total_tokens=n)) == up.UP_ERR_UNSUPPORTED


def _rotate(p=None, **kw):
    a = dict(q=A, k=A, v=A, v_stride=2 * 128, qw=A, kw=A, eps=1e-6, pos=A, freq=A, rot=128, pairs=0, count=None, q_out=A, qo=8 * 128, k_out=A,
             ko=2 * 128, v_out=A, vo=2 * 128, slots=A, num=1000)
    a.update(kw)
    return up.uniprefill_norm_rotate(p or _params(), a["q"], a["k"], a["v"], a["v_stride"], a["qw"], a["kw"], a["eps"], a["pos"], a["freq"], a["rot"],
                                     a["pairs"], a["count"], a["q_out"], a["qo"], a["k_out"], a["ko"], a["v_out"], a["vo"], a["slots"], a["num"],
                                     stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), up.UP_ERR_NULL), (dict(k_out=None), up.UP_ERR_NULL), (dict(v=None), up.UP_ERR_NULL), (dict(pos=None), up.UP_ERR_NULL),
    (dict(freq=None), up.UP_ERR_NULL), (dict(q=None, q_out=None, k=None, k_out=None, v=None, v_out=None), up.UP_ERR_NULL),
    (dict(eps=-1e-6), up.UP_ERR_RANGE), (dict(eps=NAN), up.UP_ERR_RANGE), (dict(eps=INF), up.UP_ERR_RANGE), (dict(eps=1e-41), up.UP_ERR_RANGE),
    (dict(eps=0.0), up.UP_ERR_RANGE), (dict(eps=0.0, qw=None), up.UP_ERR_RANGE), (dict(rot=-16), up.UP_ERR_RANGE), (dict(rot=144), up.UP_ERR_RANGE),
    (dict(rot=24), up.UP_ERR_UNSUPPORTED), (dict(num=-1), up.UP_ERR_SHAPE), (dict(v_stride=255), up.UP_ERR_SHAPE), (dict(qo=1000), up.UP_ERR_SHAPE),
    (dict(ko=255), up.UP_ERR_SHAPE), (dict(vo=260), up.UP_ERR_ALIGN), (dict(ko=1 << 61), up.UP_ERR_UNSUPPORTED), (dict(q=A + 8), up.UP_ERR_ALIGN),
    (dict(k_out=A + 8), up.UP_ERR_ALIGN), (dict(v_out=A + 8), up.UP_ERR_ALIGN), (dict(qw=A + 4), up.UP_ERR_ALIGN), (dict(pos=A + 2), up.UP_ERR_ALIGN),
    (dict(freq=A + 2), up.UP_ERR_ALIGN), (dict(slots=A + 4), up.UP_ERR_ALIGN), (dict(count=A + 1), up.UP_ERR_ALIGN),
])
def test_rotate_refusals(kw, want):
    assert _rotate(**kw) == want


def _pages(**kw):
    a = dict(len=A, new=A, seqs=2, page=16, table=A, tstride=8, free=A, num_free=A, left=A, new_len=A, cu=A, cuk=A, pos=A, slots=A, cap=100, served=A)
    a.update(kw)
    return up.uniprefill_append_pages(a["len"], a["new"], a["seqs"], a["page"], a["table"], a["tstride"], a["free"], a["num_free"], a["left"],
                                      a["new_len"], a["cu"], a["cuk"], a["pos"], a["slots"], a["cap"], a["served"], stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    *[({name: None}, up.UP_ERR_NULL) for name in ("len", "new", "table", "free", "num_free", "left", "new_len", "cu", "cuk", "pos", "slots", "served")],
    *[({name: A + 2}, up.UP_ERR_ALIGN) for name in ("len", "new", "table", "free", "num_free", "left", "new_len", "cu", "cuk", "pos", "served")],
    (dict(slots=A + 4), up.UP_ERR_ALIGN), (dict(seqs=-1), up.UP_ERR_SHAPE), (dict(cap=-1), up.UP_ERR_SHAPE), (dict(page=0), up.UP_ERR_RANGE),
    (dict(tstride=-1), up.UP_ERR_RANGE), (dict(cap=2 ** 31 - 2), up.UP_ERR_UNSUPPORTED), (dict(seqs=2 ** 31 - 2), up.UP_ERR_UNSUPPORTED),
    (dict(new_len=A + 4), up.UP_ERR_UNSUPPORTED), (dict(new_len=A - 4), up.UP_ERR_UNSUPPORTED),
])
def test_pages_refusals(kw, want):
    assert _pages(**kw) == want


def test_linear_plans():
    # one long sequence is cut, and the room for what its pieces add is asked for; many sequences of the same length are not
    p = _params(num_seqs=1, total_tokens=30000)
    cu = np.array([0, 30000], np.int32)
    need = up.uniprefill_linear_attention_plan(p, cu)[1]
    assert 0 < need < 1 << 30
    kw = dict(cu_host=cu, out_stride=8 * 128)
    assert _linear(p, ws=None, **kw) == up.UP_ERR_WORKSPACE
    assert _linear(p, ws_bytes=need - 1, **kw) == up.UP_ERR_WORKSPACE
    assert _linear(p, ws=A + 16, **kw) == up.UP_ERR_ALIGN
    n = 1000
    p = _params(num_seqs=n, total_tokens=50 * n, num_kv_heads=8)
    assert up.uniprefill_linear_attention_plan(p, np.arange(n + 1, dtype=np.int32) * 50)[1] == 0
    assert up.uniprefill_linear_attention_plan(p, None, check=False)[0] == up.UP_ERR_NULL
