"""CPU-only tests of the attention operators' boundary: every refusal comes back on the host before anything is
launched (there is no GPU in the process), plans are pure, and empty batches are legal."""
import ctypes

import numpy as np
import pytest

import oracle.attention_oracle as ao
import paper_2605_06221_amd as up

A = 1 << 20            # a 16- and 256-byte aligned address that is never read
L = up.lib()


def _params(**kw):
    base = dict(num_seqs=2, total_tokens=100, block_size=64, num_q_heads=8, num_kv_heads=2)
    base.update(kw)
    return up.make_params(**base)


CU = np.array([0, 60, 100], np.int32)
CK = np.array([0, 100, 200], np.int32)


def _attention(p=None, **kw):
    a = dict(q=A, k=A, v=A, v_stride=2 * 128, cu=A, cu_host=CU, cuk=None, cuk_host=None, table=None, tstride=0, page=16, out=A,
             out_stride=8 * 128, lse=A, lse_stride=100, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return up.uniprefill_attention(p or _params(), a["q"], a["k"], a["v"], a["v_stride"], a["cu"], a["cu_host"], a["cuk"],
                                   a["cuk_host"], a["table"], a["tstride"], a["page"], a["out"], a["out_stride"], a["lse"],
                                   a["lse_stride"], a["ws"], a["ws_bytes"], stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), up.UP_ERR_NULL), (dict(v=None), up.UP_ERR_NULL), (dict(out=None), up.UP_ERR_NULL), (dict(cu=None), up.UP_ERR_NULL),
    (dict(cu_host=None), up.UP_ERR_NULL), (dict(cuk=A), up.UP_ERR_NULL), (dict(table=A, tstride=99), up.UP_ERR_NULL),
    (dict(cu_host=np.array([0, 60, 99], np.int32)), up.UP_ERR_SHAPE),
    (dict(cuk=A, cuk_host=np.array([0, 59, 200], np.int32)), up.UP_ERR_SHAPE),
    (dict(cuk=A, cuk_host=CK, table=A, tstride=6), up.UP_ERR_SHAPE),
    (dict(cuk=A, cuk_host=CK, table=A, tstride=7, page=0), up.UP_ERR_RANGE),
    (dict(v_stride=2 * 128 - 8), up.UP_ERR_SHAPE), (dict(v_stride=2 * 128 + 4), up.UP_ERR_ALIGN),
    (dict(out_stride=8 * 128 - 8), up.UP_ERR_SHAPE), (dict(out_stride=8 * 128 + 4), up.UP_ERR_ALIGN),
    (dict(lse_stride=99), up.UP_ERR_SHAPE), (dict(lse=A + 2), up.UP_ERR_ALIGN),
    (dict(q=A + 8), up.UP_ERR_ALIGN), (dict(v=A + 8), up.UP_ERR_ALIGN), (dict(out=A + 8), up.UP_ERR_ALIGN),
])
def test_attention_refusals(kw, want):
    assert _attention(**kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=96), up.UP_ERR_UNSUPPORTED), (dict(num_q_heads=9), up.UP_ERR_UNSUPPORTED), (dict(num_q_heads=130), up.UP_ERR_UNSUPPORTED),
    (dict(qk_dtype=3), up.UP_ERR_UNSUPPORTED), (dict(head_dim=256, qk_dtype=up.UP_F32), up.UP_ERR_UNSUPPORTED),
    (dict(softmax_scale=-1.0), up.UP_ERR_RANGE), (dict(softmax_scale=float("nan")), up.UP_ERR_RANGE), (dict(q_row_stride=100), up.UP_ERR_SHAPE),
    (dict(k_row_stride=2 * 128 + 4), up.UP_ERR_ALIGN), (dict(num_seqs=-1), up.UP_ERR_SHAPE),
])
def test_attention_refuses_bad_parameters(kw, want):
    assert _attention(_params(**kw)) == want


def test_attention_workspace():
    # one decode token on a long cache: its keys are cut, and the room for the pieces is asked for
    p = _params(num_seqs=1, total_tokens=1)
    cu, ck = np.array([0, 1], np.int32), np.array([0, 200000], np.int32)
    st, need = up.uniprefill_attention_plan(p, cu, ck)
    assert need > 0 and need % 256 == 0
    kw = dict(cu_host=cu, cuk=A, cuk_host=ck)
    assert _attention(p, ws=None, **kw) == up.UP_ERR_WORKSPACE
    assert _attention(p, ws_bytes=need - 1, **kw) == up.UP_ERR_WORKSPACE
    assert _attention(p, ws=A + 16, **kw) == up.UP_ERR_ALIGN
    # a batch that fills the chip needs none
    p = _params(num_seqs=1, total_tokens=131072, num_q_heads=32, num_kv_heads=8)
    assert up.uniprefill_attention_plan(p, np.array([0, 131072], np.int32))[1] == 0
    # many short sequences beside one long cache: room for the long one's pieces only
    n = 3000
    p = _params(num_seqs=n + 1, total_tokens=n + 1)
    cu = np.arange(n + 2, dtype=np.int32)
    ck = np.concatenate([np.arange(n + 1, dtype=np.int32) * 20, [n * 20 + 3_000_000]]).astype(np.int32)
    assert 0 < up.uniprefill_attention_plan(p, cu, ck)[1] < 1 << 30
    assert up.uniprefill_attention_plan(_params(), CU, np.array([0, 10, 200], np.int32), check=False)[0] == up.UP_ERR_SHAPE
    assert L.uniprefill_attention_plan(ctypes.byref(_params()), up.ptr(CU), None, None) == up.UP_ERR_NULL


def test_attention_of_no_tokens():
    for lengths in ([], [0, 0, 0]):
        cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        p = _params(num_seqs=len(lengths), total_tokens=0)
        assert up.uniprefill_attention_plan(p, cu)[1] == 0
        assert _attention(p, q=None, k=None, v=None, out=None, lse=None, ws=None, ws_bytes=0, cu_host=cu) == up.UP_OK


def test_q4_row_bytes():
    for heads in (1, 3, 8):
        for d in (64, 128, 256):
            rows = ao.q4_pack(*ao.q4_quantise(np.zeros((1, heads, d), np.float32)))
            assert up.uniprefill_q4_row_bytes(heads, d) == rows.shape[1]
    assert up.uniprefill_q4_row_bytes(8, 96) == 0 and up.uniprefill_q4_row_bytes(0, 64) == 0


STORE = dict(k=A, v=A, v_stride=256, slots=A, n=10, count=None, kc=A, vc=A, stride=144, num_slots=64)


def _store(p=None, load=False, **kw):
    a = dict(STORE, **kw)
    p = p or _params()
    if load:
        return up.uniprefill_cache_load_q4(p, a["kc"], a["vc"], a["stride"], a["num_slots"], a["slots"], a["n"], a["count"], a["k"],
                                           a["v"], a["v_stride"], stream=0, check=False)
    return up.uniprefill_cache_store_q4(p, a["k"], a["v"], a["v_stride"], a["slots"], a["n"], a["count"], a["kc"], a["vc"],
                                        a["stride"], a["num_slots"], stream=0, check=False)


@pytest.mark.parametrize("load", [False, True])
@pytest.mark.parametrize("kw,want", [
    (dict(k=None), up.UP_ERR_NULL), (dict(vc=None), up.UP_ERR_NULL), (dict(k=None, kc=None, v=None, vc=None), up.UP_ERR_NULL),
    (dict(slots=None), up.UP_ERR_NULL), (dict(n=-1), up.UP_ERR_SHAPE), (dict(num_slots=-1), up.UP_ERR_SHAPE),
    (dict(v_stride=255), up.UP_ERR_SHAPE), (dict(v_stride=260), up.UP_ERR_ALIGN), (dict(stride=128), up.UP_ERR_SHAPE),
    (dict(stride=152), up.UP_ERR_ALIGN), (dict(kc=A + 8), up.UP_ERR_ALIGN), (dict(v=A + 4), up.UP_ERR_ALIGN),
    (dict(slots=A + 4), up.UP_ERR_ALIGN), (dict(count=A + 1), up.UP_ERR_ALIGN), (dict(n=1 << 31), up.UP_ERR_UNSUPPORTED),
    (dict(n=0, slots=None, k=None, v=None), up.UP_OK),
])
def test_cache_copy_refusals(kw, want, load):
    assert _store(load=load, **kw) == want
    assert _store(_params(head_dim=96), load=load) == up.UP_ERR_UNSUPPORTED


def _decode(p=None, **kw):
    a = dict(q=A, kc=A, vc=A, stride=144, len=A, max_len=100, table=A, tstride=7, page=16, out=A, out_stride=8 * 128, lse=A,
             lse_stride=2, mass_in=None, mass_out=None, mass_stride=0, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return up.uniprefill_attention_q4(p or _params(total_tokens=2), a["q"], a["kc"], a["vc"], a["stride"], a["len"], a["max_len"],
                                      a["table"], a["tstride"], a["page"], a["out"], a["out_stride"], a["lse"], a["lse_stride"],
                                      a["mass_in"], a["mass_out"], a["mass_stride"], a["ws"], a["ws_bytes"], stream=0, check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), up.UP_ERR_NULL), (dict(kc=None), up.UP_ERR_NULL), (dict(len=None), up.UP_ERR_NULL), (dict(out=None), up.UP_ERR_NULL),
    (dict(table=None), up.UP_ERR_NULL), (dict(mass_in=A), up.UP_ERR_NULL), (dict(max_len=-1), up.UP_ERR_SHAPE),
    (dict(tstride=6), up.UP_ERR_SHAPE), (dict(page=0), up.UP_ERR_RANGE), (dict(tstride=-1), up.UP_ERR_RANGE),
    (dict(stride=128), up.UP_ERR_SHAPE), (dict(stride=152), up.UP_ERR_ALIGN), (dict(out_stride=1000), up.UP_ERR_SHAPE),
    (dict(lse_stride=1), up.UP_ERR_SHAPE), (dict(mass_out=A, mass_stride=99), up.UP_ERR_SHAPE), (dict(q=A + 8), up.UP_ERR_ALIGN),
    (dict(mass_out=A + 2, mass_stride=100), up.UP_ERR_ALIGN), (dict(ws=None), up.UP_ERR_WORKSPACE), (dict(ws=A + 16), up.UP_ERR_ALIGN),
    (dict(ws_bytes=16), up.UP_ERR_WORKSPACE),
])
def test_decode_refusals(kw, want):
    assert _decode(**kw) == want


def test_decode_refuses_bad_parameters_and_plans():
    assert _decode(_params()) == up.UP_ERR_SHAPE                                     # not one token per sequence
    assert _decode(_params(total_tokens=2, qk_dtype=up.UP_F32)) == up.UP_ERR_UNSUPPORTED
    assert _decode(_params(num_seqs=0, total_tokens=0), q=None, out=None, len=None, ws=None, ws_bytes=0, table=None) == up.UP_OK
    p = _params(num_seqs=4, total_tokens=4)
    _, plain = up.uniprefill_attention_q4_plan(p, 5000, False)
    _, mass = up.uniprefill_attention_q4_plan(p, 5000, True)
    assert plain > 0 and mass >= plain + 4 * 8 * 5000 * 4 and mass % 256 == 0
    assert up.uniprefill_attention_q4_plan(_params(), 5000, False, check=False)[0] == up.UP_ERR_SHAPE
    assert up.uniprefill_attention_q4_plan(p, -1, False, check=False)[0] == up.UP_ERR_SHAPE
    assert L.uniprefill_attention_q4_plan(ctypes.byref(p), 10, 0, None) == up.UP_ERR_NULL


def _evict(**kw):
    a = dict(kc=A, vc=A, row=1024, stride=1024, mass=A, mass_stride=100, len=A, seqs=2, max_len=100, budget=50, sink=10, recent=10,
             table=A, tstride=7, new=A, nstride=4, page=16, kept=A, mass_out=A, out_stride=50, new_len=A)
    a.update(kw)
    return up.uniprefill_cache_evict(a["kc"], a["vc"], a["row"], a["stride"], a["mass"], a["mass_stride"], a["len"], a["seqs"],
                                     a["max_len"], a["budget"], a["sink"], a["recent"], a["table"], a["tstride"], a["new"],
                                     a["nstride"], a["page"], a["kept"], a["mass_out"], a["out_stride"], a["new_len"], stream=0,
                                     check=False)


@pytest.mark.parametrize("kw,want", [
    (dict(seqs=-1), up.UP_ERR_SHAPE), (dict(max_len=-1), up.UP_ERR_SHAPE), (dict(budget=0, sink=0, recent=0), up.UP_ERR_RANGE),
    (dict(budget=19), up.UP_ERR_RANGE), (dict(sink=-1), up.UP_ERR_RANGE), (dict(recent=-1), up.UP_ERR_RANGE),
    (dict(row=0), up.UP_ERR_SHAPE), (dict(row=1040), up.UP_ERR_SHAPE), (dict(row=1000), up.UP_ERR_ALIGN), (dict(stride=1032), up.UP_ERR_ALIGN),
    (dict(mass_stride=99), up.UP_ERR_SHAPE), (dict(out_stride=49), up.UP_ERR_SHAPE), (dict(kc=A + 8), up.UP_ERR_ALIGN),
    (dict(vc=A + 8), up.UP_ERR_ALIGN), (dict(kc=None), up.UP_ERR_NULL), (dict(mass=None), up.UP_ERR_NULL), (dict(len=None), up.UP_ERR_NULL),
    (dict(kept=None), up.UP_ERR_NULL), (dict(mass_out=None), up.UP_ERR_NULL), (dict(new_len=None), up.UP_ERR_NULL),
    (dict(table=None), up.UP_ERR_NULL), (dict(new=None), up.UP_ERR_NULL), (dict(tstride=6), up.UP_ERR_SHAPE), (dict(nstride=3), up.UP_ERR_SHAPE),
    (dict(page=0), up.UP_ERR_RANGE), (dict(seqs=70000), up.UP_ERR_UNSUPPORTED), (dict(mass=A + 2), up.UP_ERR_ALIGN), (dict(seqs=0), up.UP_OK),
])
def test_evict_refusals(kw, want):
    assert _evict(**kw) == want


def test_refusals_of_what_the_kernels_cannot_count():
    wide = _params(k_row_stride=(1 << 26) + 8)      # bf16: more than 2^27 bytes
    assert _attention(wide) == up.UP_ERR_UNSUPPORTED
    assert _attention(v_stride=(1 << 26) + 8) == up.UP_ERR_UNSUPPORTED
    most = (1 << 31) - 1 - 65536
    for n, want in ((most, up.UP_OK), (most + 1, up.UP_ERR_UNSUPPORTED)):
        cu, ck = np.array([0, 1], np.int32), np.array([0, n], np.int32)
        assert up.uniprefill_attention_plan(_params(num_seqs=1, total_tokens=1), cu, ck, check=False)[0] == want
        assert up.uniprefill_attention_q4_plan(_params(num_seqs=1, total_tokens=1), n, False, check=False)[0] == want
    assert _evict(max_len=most + 1, mass_stride=1 << 32, tstride=1 << 32) == up.UP_ERR_UNSUPPORTED
    # more 16-byte pieces of kept rows than are counted in 31 bits
    assert _evict(max_len=1 << 30, mass_stride=1 << 30, tstride=1 << 30, budget=1 << 30, out_stride=1 << 30, nstride=1 << 30, row=64,
                  stride=64) == up.UP_ERR_UNSUPPORTED


def test_evict_refuses_masses_in_place():
    other = dict(kept=A + 4096, mass_out=A + 8192)
    for same in (dict(other, mass_out=A), dict(other, kept=A), dict(other, kept=A + 8192)):
        assert _evict(**same) == up.UP_ERR_UNSUPPORTED


def test_evict_of_no_tokens_with_rows_beyond_what_is_counted():
    # max_kv_len 0: no row is moved, and a row's 16-byte pieces still have to fit 31 bits
    for pieces in ((1 << 31) - 1024, 1 << 32):
        assert _evict(max_len=0, row=16 * pieces, stride=16 * pieces, table=None, new=None, mass=None, kept=None,
                      mass_out=None) == up.UP_ERR_UNSUPPORTED


def test_plans_refuse_what_a_launch_cannot_count():
    # work-items of a launch are counted in 32 bits: 256 of them a work-group, one for each sequence and kv head and 128 tokens and kv head
    for n, want in ((131072, up.UP_OK), (260111, up.UP_OK), (260112, up.UP_ERR_UNSUPPORTED)):
        p = _params(num_seqs=n, total_tokens=n, num_q_heads=64, num_kv_heads=64, head_dim=64)
        cu = np.arange(n + 1, dtype=np.int32)
        assert up.uniprefill_attention_plan(p, cu, check=False)[0] == want
        refused = dict(lse=None, ws=None, ws_bytes=0, out_stride=64 * 64, v_stride=64 * 64, cu_host=cu)
        assert want == up.UP_OK or _attention(p, **refused) == want
    # and 1024 for a query head of the launch that joins the pieces of a decode step
    for heads, want in ((1 << 16) - 1, up.UP_OK), (1 << 16, up.UP_ERR_UNSUPPORTED):
        p = _params(num_seqs=1, total_tokens=1, num_q_heads=64 * heads, num_kv_heads=heads, head_dim=64)
        assert up.uniprefill_attention_q4_plan(p, 1000, False, check=False)[0] == want


def test_evict_refuses_new_lengths_that_overlap_the_old_ones():
    apart = dict(kept=A + 4096, mass_out=A + 8192, len=A + 12288, seqs=100)
    for shift in (4, -4, 396, -396):
        assert _evict(**dict(apart, new_len=A + 12288 + shift)) == up.UP_ERR_UNSUPPORTED


def test_key_offsets_that_fall_out_of_range_are_refused():
    # the difference of the last two leaves 32 bits
    ck = np.array([0, 200000, -(1 << 31)], np.int32)
    ratio = np.ones(2, np.float32)
    assert up.uniprefill_attention_plan(_params(), CU, ck, check=False)[0] == up.UP_ERR_SHAPE
    assert up.uniprefill_plan_chunked(_params(), CU, ck, ratio, check=False)[0] == up.UP_ERR_SHAPE


@pytest.mark.parametrize("stride", [(1 << 60) + 16, 1 << 61, 1 << 62])
def test_strides_whose_bytes_leave_64_bits_are_refused(stride):
    f32 = dict(qk_dtype=up.UP_F32)
    for given in (dict(q_row_stride=stride), dict(k_row_stride=stride)):
        assert _attention(_params(**given, **f32)) == up.UP_ERR_UNSUPPORTED
        assert up.uniprefill_attention_plan(_params(**given, **f32), CU, check=False)[0] == up.UP_ERR_UNSUPPORTED
    assert _attention(_params(**f32), v_stride=stride) == up.UP_ERR_UNSUPPORTED
    assert _attention(_params(**f32), out_stride=stride) == up.UP_ERR_UNSUPPORTED
    assert _decode(out_stride=stride) == up.UP_ERR_UNSUPPORTED
    for load in (False, True):
        assert _store(load=load, v_stride=stride) == up.UP_ERR_UNSUPPORTED
    p = _params(hidden_dim=64, hidden_row_stride=stride, hidden_dtype=up.UP_F32)
    assert up.uniprefill_compact(p, A, None, A, 10, A, None, stream=0, check=False) == up.UP_ERR_UNSUPPORTED


def test_the_current_stream_is_found_without_torchs_private_function(monkeypatch):
    import types

    import torch
    from paper_2605_06221_amd import binding
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=4096))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 8192 + device, raising=False)
    assert binding._stream(None).value == 8195
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert binding._stream(None).value == 4096
