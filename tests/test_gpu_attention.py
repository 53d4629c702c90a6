"""GPU tests of the attention layer's operators against the 64-bit oracle: causal attention of packed batches, the
4-bit KV cache, decode attention over it, eviction, and all of them in a row.

Tolerances (u = half a step of the type: bf16 2^-8, float 2^-24).  A logit is a float sum of D products, off by
at most d = (D + 4) 2^-24 S + 4 * 2^-24 (|x| + 1) with S = scale * sum |q k| and |x| <= S; a weight is then off by 2d
relative (its own logit and its normaliser), and an output by its own rounding, u |o|, plus what the weights' roundings
leave of A = the attention of |v|: (2d + (N + 64) 2^-24) A, and u A more where the weights are rounded to bf16."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2605_06221_amd as up
from gpu_util import host_bits
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


def _say(*a):
    print(*a, flush=True)


def _cu(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _rows(rng, dtype, *shape):
    """Normal values of the type, and the same in float64."""
    t = torch.from_numpy(rng.standard_normal(shape).astype(np.float32))
    t = t if dtype == torch.float32 else t.to(torch.bfloat16)
    return t, t.double().numpy()


def _strided(t, pad, poison):
    """t [n, H, D] as the front of wider rows on the device, the rest filled with `poison`."""
    n, h, d = t.shape
    wide = torch.full((n, h * d + pad), poison, dtype=t.dtype, device="cuda")
    wide[:, :h * d] = t.reshape(n, h * d).cuda()
    return wide


def _logit_error(S, D):
    return (D + 4) * F * S + 4 * F * (S + 1)


def _attention_tolerance(out, absv, top, n_keys, D, bf16):
    d = _logit_error(top, D).T[:, :, None]
    u = 2.0 ** -8 if bf16 else F
    return u * np.abs(out) + (2 * d + (n_keys + 64) * F + (u if bf16 else 0.0)) * absv + 1e-30


def _lse_tolerance(lse, top, n_keys, D):
    return _logit_error(top, D) + (n_keys + 64) * F + 4 * F * (np.abs(lse) + 1)


class Batch:
    """A packed batch with everything that a call of uniprefill_attention takes."""

    def __init__(self, seed, lengths, hq, hkv, D, dtype=torch.bfloat16, earlier=None, page=0, pad=0, scale=0.0, key_scale=1.0):
        rng = np.random.default_rng(seed)
        self.lengths, self.D, self.dtype, self.page = lengths, D, dtype, page
        self.keys = [n + e for n, e in zip(lengths, earlier or [0] * len(lengths))]
        self.cu_host, self.ck_host = _cu(lengths), _cu(self.keys)
        T, Tk = int(self.cu_host[-1]), int(self.ck_host[-1])
        q, self.q64 = _rows(rng, dtype, T, hq, D)
        k, k64 = _rows(rng, dtype, Tk, hkv, D)
        if key_scale != 1.0:
            k = k * key_scale
            k64 = k.double().numpy()
        v, v64 = _rows(rng, dtype, Tk, hkv, D)
        self.ctx = earlier is not None
        self.gather, self.table, self.tstride = None, None, 0
        nan = float("nan")
        if page:
            need = [-(-n // page) for n in self.keys]
            order = rng.permutation(sum(need) + 2)
            table = np.full((len(lengths), max(need + [1]) + 1), -1, np.int32)
            at = 0
            for r, n in enumerate(need):
                table[r, :n] = order[at:at + n]
                at += n
            kc, vc = (torch.full(((sum(need) + 2) * page, hkv, D), nan, dtype=dtype) for _ in range(2))
            for r, n in enumerate(self.keys):
                at = ao.page_rows(table[r], n, page)
                kc[at], vc[at] = k[self.ck_host[r]:self.ck_host[r + 1]], v[self.ck_host[r]:self.ck_host[r + 1]]
            k, v = kc, vc
            k64, v64 = k.double().numpy(), v.double().numpy()
            self.gather = lambda r, n: ao.page_rows(table[r], n, page)
            self.table, self.tstride = _dev(table), table.shape[1]
        self.k64, self.v64 = k64, v64
        self.q, self.k, self.v = (_strided(t, pad, nan) for t in (q, k, v))
        self.out = torch.full((T + 3, hq * D + pad), -7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((hq, T + 5), -7.0, device="cuda")
        self.cu, self.ck = _dev(self.cu_host), _dev(self.ck_host)
        self.scale = scale
        self.p = up.make_params(num_seqs=len(lengths), total_tokens=T, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                                q_row_stride=hq * D + pad, k_row_stride=hkv * D + pad, softmax_scale=scale,
                                qk_dtype=up.UP_F32 if dtype == torch.float32 else up.UP_BF16)
        _, self.ws_bytes = up.uniprefill_attention_plan(self.p, self.cu_host, self.ck_host if self.ctx else None)
        self.ws = torch.full((self.ws_bytes + 256,), 255, dtype=torch.uint8, device="cuda")

    def run(self, want_lse=True, stream=None):
        return up.uniprefill_attention(
            self.p, self.q, self.k, self.v, self.v.shape[1], self.cu, self.cu_host, self.ck if self.ctx else None,
            self.ck_host if self.ctx else None, self.table, self.tstride, max(self.page, 1), self.out, self.out.shape[1],
            self.lse if want_lse else None, self.lse.shape[1], self.ws, self.ws_bytes, stream=stream)

    def results(self):
        torch.cuda.synchronize()
        T, hq = int(self.cu_host[-1]), self.lse.shape[0]
        return (self.out[:T, :hq * self.D].double().cpu().numpy().reshape(T, hq, self.D), self.lse[:, :T].double().cpu().numpy())

    def check(self, want_lse=True):
        T, hq = int(self.cu_host[-1]), self.lse.shape[0]
        want, lse, absv, top = ao.causal_attention(self.q64, self.k64, self.v64, self.cu_host, self.ck_host,
                                                   scale=self.scale or None, gather=self.gather)
        got, got_lse = self.results()
        n = max(self.keys + [1])
        tol = _attention_tolerance(want, absv, top, n, self.D, self.dtype == torch.bfloat16)
        worst = np.max(np.abs(got - want) / tol) if T else 0.0
        _say("  worst error / tolerance", float(worst))
        assert worst <= 1.0, np.unravel_index(np.argmax(np.abs(got - want) / tol), got.shape)
        if want_lse:
            assert (np.abs(got_lse - lse) <= _lse_tolerance(lse, top, n, self.D)).all()
        else:
            assert (self.lse == -7.0).all()
        assert (self.out[T:] == -7.0).all() and (self.out[:, hq * self.D:] == -7.0).all() and (self.lse[:, T:] == -7.0).all()


BF, F32 = torch.bfloat16, torch.float32
SHAPES = [      # lengths, q heads, kv heads, head dimension, type
    ([1], 1, 1, 64, BF), ([1, 0, 2, 63, 64, 65], 8, 2, 64, BF), ([129, 31, 1, 500], 8, 8, 128, BF), ([777], 40, 8, 128, BF),
    ([300, 0, 0, 41], 5, 1, 128, BF), ([130, 7], 64, 1, 128, BF), ([200, 33, 95], 6, 2, 256, BF), ([1025], 4, 4, 256, BF),
    ([0, 1, 64, 130], 8, 2, 64, F32), ([333, 1], 10, 2, 128, F32), ([65], 3, 3, 128, F32), ([1] * 40, 12, 4, 128, BF),
]


@pytest.mark.parametrize("lengths,hq,hkv,D,dtype", SHAPES)
def test_attention_of_whole_prompts(lengths, hq, hkv, D, dtype):
    _say("attention", lengths, hq, hkv, D, dtype)
    b = Batch(len(lengths) * D + hq, lengths, hq, hkv, D, dtype)
    b.run()
    b.check()


@pytest.mark.parametrize("page", [0, 1, 7, 16, 48])
@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (128, F32)])
def test_attention_after_earlier_context(page, D, dtype):
    _say("attention after context", page, D, dtype)
    b = Batch(page + D, [5, 1, 0, 140, 33], 8, 2, D, dtype, earlier=[700, 1300, 9, 0, 61], page=page, pad=16)
    b.run()
    b.check()


@pytest.mark.parametrize("lengths,earlier,hq,hkv,D,dtype", [
    ([1], [20000], 8, 1, 128, BF), ([1, 1, 3], [5000, 1, 9000], 4, 4, 64, BF), ([40, 1], [4000, 2500], 8, 2, 256, BF),
    ([2], [6000], 64, 1, 128, BF), ([1, 30], [3000, 2100], 5, 5, 128, F32), ([1] * 300 + [2], [3] * 300 + [9000], 4, 4, 64, BF),
])
def test_attention_with_the_keys_cut_into_pieces(lengths, earlier, hq, hkv, D, dtype):
    _say("attention in pieces", lengths[:4], earlier[:4], hq, hkv, D, dtype)
    for page in (0, 16):
        b = Batch(7, lengths, hq, hkv, D, dtype, earlier=earlier, page=page)
        assert b.ws_bytes > 0
        b.run()
        b.check()


@pytest.mark.parametrize("lengths,earlier,hq,hkv,D,dtype,page", [
    ([2100, 1, 67], None, 32, 8, 128, BF, 0), ([1100], [333], 64, 8, 64, BF, 16), ([700, 0, 400], [50, 0, 0], 64, 8, 256, BF, 8),
    ([1010], [129], 64, 16, 128, F32, 24), ([1010, 1], [3, 2500], 64, 16, 64, F32, 7), ([2100, 1], [0, 30000], 32, 8, 128, BF, 16),
    ([1050, 3], [0, 9000], 64, 8, 64, BF, 0), ([1050, 2], [100, 5000], 64, 16, 256, BF, 5),
    # two rounds and more
    ([300], [700], 512, 8, 128, BF, 16), ([520, 1, 67], None, 256, 16, 64, BF, 0), ([600, 0, 30], [40, 0, 9000], 256, 16, 256, BF, 8),
    ([530], [129], 256, 16, 128, F32, 24), ([530, 1], [3, 2500], 256, 16, 64, F32, 7), ([1100], None, 128, 32, 128, BF, 0),
    ([540, 2], [100, 5000], 256, 16, 256, BF, 5), ([270, 1], [0, 30000], 512, 8, 64, BF, 128), ([515], None, 256, 16, 128, F32, 0),
    ([515], None, 256, 16, 64, F32, 0), ([515], None, 256, 16, 256, BF, 0), ([140, 140], [2000, 1999], 512, 8, 128, BF, 0),
])
def test_attention_in_work_groups_of_256_rows(lengths, earlier, hq, hkv, D, dtype, page):
    """Batches with at least as many tiles of 256 rows as the chip has CUs: eight waves per work-group, or four where one round of them
    would be uneven."""
    _say("attention, large", lengths, earlier, hq, hkv, D, dtype, page)
    assert sum(-(-n * (hq // hkv) // 256) for n in lengths) * hkv >= 256
    b = Batch(31, lengths, hq, hkv, D, dtype, earlier=earlier, page=page)
    b.run()
    b.check()


def test_attention_strides_scale_and_no_lse():
    _say("attention: padded rows (NaN in the padding), softmax scale, no log-sum-exp")
    b = Batch(3, [100, 37], 8, 2, 128, pad=24, scale=0.3)
    b.run(want_lse=False)
    b.check(want_lse=False)


@pytest.mark.parametrize("key_scale", [0.0, 30.0])
def test_attention_of_flat_and_of_concentrated_rows(key_scale):
    # all logits equal (a mean of the visible values), and logits of some hundred (one key takes all the weight)
    _say("attention, keys times", key_scale)
    b = Batch(5, [260, 90], 4, 2, 128, key_scale=key_scale)
    b.run()
    b.check()


def test_attention_is_the_same_on_every_run_and_on_another_stream():
    _say("attention: runs and streams")
    b = Batch(11, [1, 400, 2], 8, 2, 128, earlier=[9000, 100, 0], page=16)
    b.run()
    first = b.results()
    side = torch.cuda.Stream()
    for i in range(5):
        b.out.fill_(-7.0)
        b.ws.fill_(i)
        torch.cuda.synchronize()
        b.run(stream=side if i % 2 else None)
        again = b.results()
        np.testing.assert_array_equal(first[0], again[0])
        np.testing.assert_array_equal(first[1], again[1])


def _graph(call):
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    return g


def test_calls_without_a_stream_go_to_the_current_one():
    from paper_2605_06221_amd import binding
    for side in (torch.cuda.default_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(side):
            assert (binding._stream(None).value or 0) == side.cuda_stream


def test_attention_and_decode_replayed_from_a_graph():
    _say("graphs: attention in pieces, decode with masses, two graphs in turn on one workspace each")
    b = Batch(12, [1, 300], 8, 2, 128, earlier=[5000, 0])
    d = Decode(13, [500, 12, 77], 8, 2, 128, mass=True)
    ga, gd = _graph(b.run), _graph(d.run)
    rng = np.random.default_rng(1)
    for i in range(4):
        q, b.q64 = _rows(rng, BF, *b.q64.shape)
        b.q[:, :q.shape[1] * q.shape[2]] = q.reshape(q.shape[0], -1).cuda()
        q, d.q64 = _rows(rng, BF, *d.q64.shape)
        d.q[:, :q.shape[1] * q.shape[2]] = q.reshape(q.shape[0], -1).cuda()
        d.set_lengths([500 - 100 * i, 4 * i, 0 if i == 2 else 77])      # (never longer than the pages there are)
        b.out.fill_(-7.0)
        d.out.fill_(-7.0)
        d.mass_out.fill_(-7.0)
        ga.replay()
        gd.replay()
        b.check()
        d.check()


# ----------------------------------------------------------------------------- the 4-bit cache
def _copy_params(heads, D, dtype, pad=0):
    return up.make_params(num_seqs=1, total_tokens=1, block_size=64, num_q_heads=heads, num_kv_heads=heads, head_dim=D,
                          k_row_stride=heads * D + pad, qk_dtype=up.UP_F32 if dtype == F32 else up.UP_BF16)


def _hard_rows(rng, dtype, n, heads, D):
    """Rows with equal elements, zeros, ties of the rounding, tiny and huge ranges, one outlier."""
    x = rng.standard_normal((n, heads, D)).astype(np.float32)
    x *= np.exp(4 * rng.standard_normal((n, heads, 1))).astype(np.float32)
    kinds = [np.zeros(D), np.full(D, -3.25), np.arange(D) % 31 * 0.5 - 2, np.where(np.arange(D) % 64 == 5, 1e30, 1.0),
             1e-30 * np.arange(D), np.where(np.arange(D) % 2 == 0, 3e38, -3e38), -np.arange(D) / 1024.0, np.full(D, 1e-38),
             np.where(np.arange(D) % 3 == 0, 1e-39, 0.0)]
    for i in range(min(n, 2 * len(kinds))):
        x[i, i % heads] = kinds[i % len(kinds)].astype(np.float32)
    t = torch.from_numpy(x)
    return t if dtype == F32 else t.to(BF)


@pytest.mark.parametrize("n,heads,D,dtype", [(1, 1, 64, BF), (3, 3, 64, F32), (77, 8, 128, BF), (50, 5, 128, F32), (33, 2, 256, BF),
                                             (1000, 4, 64, BF), (19, 64, 128, BF)])
def test_rows_enter_and_leave_the_cache(n, heads, D, dtype):
    """Cache bytes equal the oracle's, bit for bit; so do the values that come back, rounded once."""
    _say("4-bit store and load", n, heads, D, dtype)
    rng = np.random.default_rng(n)
    k, v = _hard_rows(rng, dtype, n, heads, D), _hard_rows(rng, dtype, n, heads, D)
    pad, slots_n = 16, 2 * n + 3
    row = up.uniprefill_q4_row_bytes(heads, D)
    stride = -(-row // 16) * 16 + 16
    slots = rng.permutation(slots_n)[:n].astype(np.int64)
    skip = rng.random(n) < 0.2
    slots_given = slots.copy()
    slots_given[skip] = rng.choice([-1, slots_n, 1 << 40, -(1 << 50)], skip.sum())
    p = _copy_params(heads, D, dtype, pad)
    kd, vd = _strided(k, pad, float("nan")), _strided(v, pad, float("nan"))
    kc, vc = (torch.full((slots_n, stride), 0xAA, dtype=torch.uint8, device="cuda") for _ in range(2))
    up.uniprefill_cache_store_q4(p, kd, vd, heads * D + pad, _dev(slots_given), n, None, kc, vc, stride, slots_n)
    ko, vo = (torch.full((n + 2, heads * D + pad), -7.0, dtype=dtype, device="cuda") for _ in range(2))
    up.uniprefill_cache_load_q4(p, kc, vc, stride, slots_n, _dev(slots_given), n, None, ko, vo, heads * D + pad)
    torch.cuda.synchronize()
    for x, cache, out in ((k, kc, ko), (v, vc, vo)):
        code, lo, step = ao.q4_quantise(x.float().numpy())
        want = np.full((slots_n, stride), 0xAA, np.uint8)
        want[slots[~skip], :row] = ao.q4_pack(code, lo, step)[~skip]
        np.testing.assert_array_equal(cache.cpu().numpy(), want)
        values = torch.from_numpy(ao.q4_values(code, lo, step).astype(np.float32)).to(dtype).reshape(n, -1)
        got = out.cpu()
        # (the reference's detour over float may move a value to the neighbour of the type: one step)
        assert ((got[:n, :heads * D].double() - values.double()).abs()[~skip] <= torch.finfo(dtype).eps * values.double().abs()[~skip]).all()
        assert (got[:n, :heads * D][torch.from_numpy(skip)] == -7.0).all()
        assert (got[n:] == -7.0).all() and (got[:, heads * D:] == -7.0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["plain", "coarse", "shifted", "whole_numbers", "tiny_lowest", "no_negatives", "tiny_beside_large", "powers"])
def test_codes_next_to_ties_and_rounded_differences(kind, dtype):
    """Bit for bit the oracle's bytes where quotients are ties or nearly, and where x - lowest is not a float."""
    _say("4-bit codes", kind, dtype)
    rng = np.random.default_rng(len(kind))
    n, heads, D = 512, 4, 128
    x = rng.standard_normal((n, heads, D)).astype(np.float32)
    small = np.float32(2.0) ** rng.integers(-30, -10, x.shape)
    x = {"plain": x, "coarse": np.round(x * 4) / 4, "shifted": x + 100, "whole_numbers": rng.integers(-8, 9, x.shape),
         "tiny_lowest": np.where(np.arange(D) % 64 == 17, small, np.abs(x) + 1), "no_negatives": np.maximum(x, 0),
         "tiny_beside_large": np.where(rng.random(x.shape) < 0.1, x * small, x), "powers": small * np.sign(x)}[kind]
    t = torch.from_numpy(np.asarray(x, np.float32)).to(dtype)
    row = up.uniprefill_q4_row_bytes(heads, D)
    cache = torch.zeros(n, row, dtype=torch.uint8, device="cuda")
    up.uniprefill_cache_store_q4(_copy_params(heads, D, dtype, 0), t.cuda(), None, heads * D, _dev(np.arange(n)), n, None, cache, None, row, n)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(cache.cpu().numpy(), ao.q4_pack(*ao.q4_quantise(t.float().numpy())))


def test_cache_copies_stop_at_the_count_on_the_device():
    _say("4-bit store and load: device count, keys alone")
    rng = np.random.default_rng(0)
    n, heads, D = 21, 2, 128
    p, stride = _copy_params(heads, D, BF), 144
    k = _hard_rows(rng, BF, n, heads, D).cuda()
    slots = _dev(np.arange(n, dtype=np.int64))
    for count in (0, 13, 40):
        kc = torch.full((n, stride), 0xAA, dtype=torch.uint8, device="cuda")
        out = torch.full((n, heads, D), -7.0, dtype=BF, device="cuda")
        dev = torch.tensor([count], dtype=torch.int32, device="cuda")
        up.uniprefill_cache_store_q4(p, k, None, heads * D, slots, n, dev, kc, None, stride, n)
        up.uniprefill_cache_load_q4(p, kc, None, stride, n, slots, n, dev, out, None, heads * D)
        m = min(n, count)
        want = ao.q4_pack(*ao.q4_quantise(k.float().cpu().numpy()))
        np.testing.assert_array_equal(kc[:m].cpu().numpy(), want[:m])
        assert (kc[m:] == 0xAA).all() and (out[m:] == -7.0).all() and (out[:m] != -7.0).any() == (m > 0)


# ----------------------------------------------------------------------------- decode
class Decode:
    def __init__(self, seed, lengths, hq, hkv, D, page=16, mass=False, pad=0, max_len=None, in_place=False, scale=0.0):
        rng = np.random.default_rng(seed)
        self.D, self.hkv, self.page, self.scale = D, hkv, page, scale
        R = len(lengths)
        self.max_len = max(lengths + [0]) if max_len is None else max_len
        need = [-(-n // page) for n in lengths]
        order = rng.permutation(sum(need) + 1)
        self.table_host = np.full((R, -(-self.max_len // page) + 1), -1, np.int32)      # (nothing past a length is looked up)
        at = 0
        for r, n in enumerate(need):
            self.table_host[r, :n] = order[at:at + n]
            at += n
        row = up.uniprefill_q4_row_bytes(hkv, D)
        self.stride = -(-row // 16) * 16 + 16
        self.caches, self.host = [], []
        for _ in range(2):
            # a slot that no sequence owns, and what pads a row: NaN pairs and arbitrary codes
            host = np.full(((sum(need) + 1) * page, self.stride), 0xFF, np.uint8)
            for r, n in enumerate(lengths):
                host[ao.page_rows(self.table_host[r], n, page), :row] = ao.q4_pack(
                    *ao.q4_quantise(_rows(rng, BF, n, hkv, D)[0].float().numpy())) if n else 0
            self.host.append(host)
            self.caches.append(_dev(host))
        q, self.q64 = _rows(rng, BF, R, hq, D)
        self.q = _strided(q, pad, float("nan"))
        self.out = torch.full((R + 2, hq * D + pad), -7.0, dtype=BF, device="cuda")
        self.lse = torch.full((hq, R + 3), -7.0, device="cuda")
        self.mass_in = self.mass_out = None
        if mass:
            self.mass_in = torch.from_numpy(rng.random((R, self.max_len + 5)).astype(np.float32)).cuda()
            self.mass_out = self.mass_in if in_place else torch.full_like(self.mass_in, -7.0)
            self.mass_host = self.mass_in.double().cpu().numpy()
        self.table = _dev(self.table_host)
        self.p = up.make_params(num_seqs=R, total_tokens=R, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                                q_row_stride=hq * D + pad, softmax_scale=scale)
        _, self.ws_bytes = up.uniprefill_attention_q4_plan(self.p, self.max_len, mass)
        self.ws = torch.full((self.ws_bytes + 256,), 255, dtype=torch.uint8, device="cuda")
        self.kv_len = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.set_lengths(lengths)

    def set_lengths(self, lengths, given=None):
        self.lengths = lengths
        self.kv_len.copy_(torch.tensor(given or lengths, dtype=torch.int32))

    def run(self, stream=None, mass_in=True):
        m = self.mass_out is not None
        return up.uniprefill_attention_q4(
            self.p, self.q, self.caches[0], self.caches[1], self.stride, self.kv_len, self.max_len, self.table, self.table.shape[1],
            self.page, self.out, self.out.shape[1], self.lse, self.lse.shape[1], self.mass_in if m and mass_in else None, self.mass_out,
            self.mass_out.shape[1] if m else 0, self.ws, self.ws_bytes, stream=stream)

    def check(self, mass_in=True):
        torch.cuda.synchronize()
        R, hq, D = self.q64.shape
        got = self.out[:R, :hq * D].double().cpu().numpy().reshape(R, hq, D)
        got_lse = self.lse[:, :R].double().cpu().numpy()
        worst = 0.0
        for r, n in enumerate(self.lengths):
            rows = ao.page_rows(self.table_host[r], n, self.page)
            want, lse, mean, W, near, far, top = ao.decode_attention_q4(self.q64[r], self.host[0][rows], self.host[1][rows], self.hkv,
                                                                        scale=self.scale or None)
            if n == 0:
                assert (got[r] == 0).all() and (got_lse[:, r] == -np.inf).all()
            else:
                d = _logit_error(top, D)
                tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -8 * near + (2 * d[:, None] + (n + 64) * F) * far + 1e-30
                worst = max(worst, float(np.max(np.abs(got[r] - want) / tol)))
                assert (np.abs(got_lse[:, r] - lse) <= d + (n + 64) * F + 4 * F * (np.abs(lse) + 1)).all()
            if self.mass_out is not None:
                got_mass = self.mass_out[r].double().cpu().numpy()
                base = self.mass_host[r] if mass_in else np.zeros_like(self.mass_host[r])
                if n:
                    rel = (2 * d + (2 * n + 64 + hq) * F).max()
                    assert (np.abs(got_mass[:n] - base[:n] - mean) <= rel * mean + 2 * F * (base[:n] + mean)).all()
                left = self.mass_host[r][n:] if self.mass_out is self.mass_in else -7.0
                assert (got_mass[n:] == left).all()
        _say("  worst error / tolerance", worst)
        assert worst <= 1.0
        assert (self.out[R:] == -7.0).all() and (self.out[:, hq * D:] == -7.0).all() and (self.lse[:, R:] == -7.0).all()


@pytest.mark.parametrize("lengths,hq,hkv,D,page", [
    ([1], 1, 1, 64, 16), ([1, 0, 63, 64, 65, 300], 8, 8, 128, 16), ([700, 3], 32, 8, 128, 1), ([129, 500], 40, 8, 128, 7),
    ([400], 64, 1, 128, 16), ([90, 2000], 20, 1, 64, 32), ([0, 0], 8, 2, 128, 16), ([333, 64], 6, 2, 256, 16), ([70], 9, 3, 64, 48),
    ([257, 1, 12], 16, 16, 256, 16), ([600, 40], 12, 12, 64, 128), ([5000], 10, 5, 128, 16), ([100, 9], 34, 2, 256, 16),
])
@pytest.mark.parametrize("mass", [False, True])
def test_decode_over_the_cache(lengths, hq, hkv, D, page, mass):
    _say("decode", lengths, hq, hkv, D, page, mass)
    d = Decode(hq * D, lengths, hq, hkv, D, page, mass=mass, pad=16 if mass else 0)
    d.run()
    d.check()


@pytest.mark.parametrize("R,hq,hkv,D", [(1100, 4, 2, 64), (513, 8, 8, 128), (600, 8, 4, 256)])
def test_decode_of_more_sequences_than_a_work_group_has_threads(R, hq, hkv, D):
    _say("decode: many sequences", R, hq, hkv, D)
    rng = np.random.default_rng(R)
    lengths = [int(n) for n in np.where(rng.random(R) < 0.2, 0, rng.integers(1, 200, R))]
    lengths[-1] = 77
    d = Decode(R, lengths, hq, hkv, D, mass=True)
    d.run()
    d.check()


def test_decode_lengths_beyond_the_ends_count_as_the_ends():
    _say("decode: lengths out of range, room for longer caches than there are")
    d = Decode(4, [200, 0, 200], 8, 2, 128, mass=True, max_len=200)
    d.set_lengths([200, 0, 200], given=[1 << 30, -5, 200])
    d.run()
    d.check()
    d = Decode(5, [30, 5], 8, 2, 128, mass=True, max_len=40000)
    d.run()
    d.check()


def test_decode_adds_weights_in_place_and_from_nothing():
    _say("decode: masses in place, masses from nothing")
    d = Decode(6, [100, 900], 8, 2, 128, mass=True, in_place=True)
    d.run()
    d.check()
    d = Decode(6, [100, 900], 8, 2, 128, mass=True)
    d.run(mass_in=False)
    d.check(mass_in=False)


def test_decode_is_the_same_on_every_run_and_on_another_stream():
    _say("decode: runs and streams")
    d = Decode(8, [3000, 17, 0, 800], 32, 8, 128, mass=True, scale=0.2)
    d.run()
    d.check()
    first = [t.clone() for t in (d.out, d.lse, d.mass_out)]
    side = torch.cuda.Stream()
    for i in range(4):
        d.ws.fill_(i)
        torch.cuda.synchronize()
        d.run(stream=side if i % 2 else None)
        torch.cuda.synchronize()
        for a, b in zip(first, (d.out, d.lse, d.mass_out)):
            assert torch.equal(a, b)


# ----------------------------------------------------------------------------- eviction
def _mass(rng, kind, n):
    if kind == "ties":
        return rng.integers(0, 3, n).astype(np.float32)
    if kind == "zeros":
        return np.where(rng.random(n) < 0.5, np.float32(0.0), np.float32(-0.0))
    if kind == "spread":
        return np.exp(20 * rng.standard_normal(n)).astype(np.float32)
    return np.float32(1) + np.arange(n, dtype=np.float32) * np.float32(2.0 ** -20)      # keys that differ in their last bits


@pytest.mark.parametrize("kind", ["ties", "zeros", "spread", "last_bits"])
@pytest.mark.parametrize("lengths,budget,n_sink,n_recent,page,row_bytes", [
    ([1], 1, 0, 0, 16, 16), ([5, 0, 64, 65, 1000], 64, 4, 4, 16, 144), ([3000, 10, 2049], 300, 128, 128, 7, 576),
    ([100], 100, 50, 50, 16, 32), ([101, 500], 100, 50, 50, 1, 1040), ([20000, 16385], 5000, 0, 1, 32, 64), ([700], 699, 3, 0, 16, 32),
    ([64], 1, 1, 0, 16, 16),
    # long ones: many work-groups to a sequence, without a choice to make, with one token too little room for it; one work-group and masses
    # of one first digit beyond what its LDS holds
    ([60000, 24577, 0, 9, 8999, 30000], 9000, 4, 100, 64, 16), ([40000, 12000], 12000, 6000, 6000, 128, 16), ([24576], 6164, 0, 0, 16, 16),
    ([24576], 6163, 0, 0, 16, 16), ([70000, 30000], 300, 16, 16, 64, 16), ([70000, 26000], 25500, 0, 0, 64, 16),
])
def test_eviction(lengths, budget, n_sink, n_recent, page, row_bytes, kind):
    _say("eviction", lengths, budget, n_sink, n_recent, page, row_bytes, kind)
    rng = np.random.default_rng(budget)
    R, most = len(lengths), max(lengths)
    kept = [min(n, budget) for n in lengths]
    old, new = [-(-n // page) for n in lengths], [-(-n // page) for n in kept]
    pages = rng.permutation(sum(old) + sum(new) + 1)
    table, new_table = np.full((R, max(old + [1])), -1, np.int32), np.full((R, -(-min(budget, most) // page) + 1), -1, np.int32)
    at = 0
    for t, need in ((table, old), (new_table, new)):
        for r, n in enumerate(need):
            t[r, :n] = pages[at:at + n]
            at += n
    stride = row_bytes + 32
    caches = [rng.integers(0, 256, ((at + 1) * page, stride)).astype(np.uint8) for _ in range(2)]
    mass = np.stack([_mass(rng, kind, most + 3) for _ in range(R)])
    dev = [_dev(c) for c in caches]
    kept_idx = torch.full((R, budget + 4), -77, dtype=torch.int32, device="cuda")
    mass_out = torch.full((R, budget + 4), -7.0, device="cuda")
    new_len = torch.full((R + 2,), -77, dtype=torch.int32, device="cuda")
    for v in (True, False):
        up.uniprefill_cache_evict(dev[0], dev[1] if v else None, row_bytes, stride, _dev(mass), most + 3,
                                  torch.tensor(lengths, dtype=torch.int32, device="cuda"), R, most, budget, n_sink, n_recent, _dev(table),
                                  table.shape[1], _dev(new_table), new_table.shape[1], page, kept_idx, mass_out, budget + 4, new_len)
    torch.cuda.synchronize()
    want = [c.copy() for c in caches]
    for r, n in enumerate(lengths):
        stay = ao.evict_tokens(mass[r], n, budget, n_sink, n_recent)
        m = len(stay)
        assert int(new_len[r]) == m
        np.testing.assert_array_equal(kept_idx[r, :m].cpu().numpy(), stay)
        np.testing.assert_array_equal(mass_out[r, :m].cpu().numpy(), mass[r][stay])
        assert (kept_idx[r, m:] == -77).all() and (mass_out[r, m:] == -7.0).all()
        src, dst = ao.page_rows(table[r], n, page)[stay], ao.page_rows(new_table[r], m, page)
        for w, c in zip(want, caches):
            w[dst, :row_bytes] = c[src, :row_bytes]
    assert (new_len[R:] == -77).all()
    for d, w in zip(dev, want):
        np.testing.assert_array_equal(d.cpu().numpy(), w)


# ----------------------------------------------------------------------------- all of them, as they are used
def test_eviction_clamps_lengths_of_the_device():
    _say("eviction: lengths out of range")
    rng = np.random.default_rng(51)
    n, budget, page = 600, 100, 32
    table = np.arange(3 * 19, dtype=np.int32).reshape(3, 19)
    new_table = 57 + np.arange(3 * 4, dtype=np.int32).reshape(3, 4)
    before = rng.integers(0, 256, (69 * page, 48)).astype(np.uint8)
    cache, mass = _dev(before), rng.random((3, n)).astype(np.float32)
    kept_idx, mass_out = torch.full((3, budget), -77, dtype=torch.int32, device="cuda"), torch.full((3, budget), -7.0, device="cuda")
    new_len = torch.full((3,), -77, dtype=torch.int32, device="cuda")
    up.uniprefill_cache_evict(cache, None, 48, 48, _dev(mass), n, _dev(np.array([1 << 30, -5, 70], np.int32)), 3, n, budget, 8, 8, _dev(table), 19,
                              _dev(new_table), 4, page, kept_idx, mass_out, budget, new_len)
    torch.cuda.synchronize()
    assert new_len.tolist() == [100, 0, 70] and (kept_idx[1] == -77).all() and (kept_idx[2, 70:] == -77).all()
    want = before.copy()
    for r, length in ((0, n), (2, 70)):
        stay = ao.evict_tokens(mass[r], length, budget, 8, 8)
        np.testing.assert_array_equal(kept_idx[r, :len(stay)].cpu().numpy(), stay)
        want[ao.page_rows(new_table[r], len(stay), page)] = before[ao.page_rows(table[r], length, page)[stay]]
    np.testing.assert_array_equal(cache.cpu().numpy(), want)


def test_calls_at_the_same_time_on_two_streams():
    """Two batches, two workspaces, two streams, nothing between the calls: the results of each alone."""
    _say("two streams at once")
    work = [Batch(61, [900, 70], 8, 2, 128, earlier=[3000, 0], page=16), Batch(62, [1, 1, 1], 32, 8, 128, earlier=[9000, 5000, 20]),
            Decode(63, [5000, 30, 700], 32, 8, 128, mass=True), Decode(64, [300] * 20, 8, 4, 64, mass=True)]
    alone = []
    for w in work:
        w.run()
        w.check()
        alone.append([t.clone() for t in (w.out, w.lse) + ((w.mass_out,) if isinstance(w, Decode) else ())])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(10):
        for j, w in enumerate(work):
            w.run(stream=streams[j % 2])
    torch.cuda.synchronize()
    for w, want in zip(work, alone):
        for a, b in zip((w.out, w.lse) + ((w.mass_out,) if isinstance(w, Decode) else ()), want):
            assert torch.equal(a, b)


def test_slots_beyond_4_gib_of_a_cache():
    """The same calls with their pages at the front and at the far end of caches of 4.5 GiB: the same bits."""
    _say("caches of more than 4 GiB")
    rng = np.random.default_rng(41)
    heads, hq, D, page, n, budget = 8, 16, 128, 16, 500, 200
    used, new = -(-n // page), -(-budget // page)
    mass_host = _dev(rng.random((1, n)).astype(np.float32))
    rows = _rows(rng, BF, n, heads, D)[0].cuda()
    q = _rows(rng, BF, 1, hq, D)[0].cuda()
    lens = _dev(np.array([n], np.int32))
    cu, ck = np.array([0, 1], np.int32), np.array([0, n], np.int32)
    for stride, q4 in ((heads * D * 2, False), (up.uniprefill_q4_row_bytes(heads, D), True)):
        pages = (9 << 29) // (stride * page)
        cache = torch.zeros(pages * page, stride, dtype=torch.uint8, device="cuda")
        found = []
        for first in (0, pages - used - new):
            order = first + rng.permutation(used + new)
            table, new_table = order[None, :used].astype(np.int32), order[None, used:].astype(np.int32)
            slots = ao.page_rows(table[0], n, page)
            p = up.make_params(num_seqs=1, total_tokens=1, block_size=64, num_q_heads=hq, num_kv_heads=heads, head_dim=D)
            out, lse = torch.zeros(1, hq * D, dtype=BF, device="cuda"), torch.zeros(hq, 1, device="cuda")
            tab, new_tab = _dev(table), _dev(new_table)
            ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
            if q4:
                up.uniprefill_cache_store_q4(p, rows, rows, heads * D, _dev(slots), n, None, cache, cache, stride, pages * page)
                up.uniprefill_attention_q4(p, q, cache, cache, stride, lens, n, tab, used, page, out, hq * D, lse, 1, None, None, 0, ws,
                                           ws.numel())
            else:
                cache[_dev(slots)] = rows.view(torch.uint8).reshape(n, stride)
                up.uniprefill_attention(p, q, cache, cache, heads * D, _dev(cu), cu, _dev(ck), ck, tab, used, page, out, hq * D, lse, 1,
                                        ws, ws.numel())
            kept_idx, mass_out = torch.zeros(1, budget, dtype=torch.int32, device="cuda"), torch.zeros(1, budget, device="cuda")
            new_len = torch.zeros(1, dtype=torch.int32, device="cuda")
            up.uniprefill_cache_evict(cache, None, stride, stride, mass_host, n, lens, 1, n, budget, 4, 4, tab, used, new_tab, new,
                                      page, kept_idx, mass_out, budget, new_len)
            torch.cuda.synchronize()
            moved = cache[_dev(ao.page_rows(new_table[0], budget, page))]
            assert torch.equal(moved, cache[_dev(slots)][kept_idx[0].long()]) and moved.any()
            back = torch.zeros(n, heads * D, dtype=BF, device="cuda")
            if q4:
                up.uniprefill_cache_load_q4(p, cache, None, stride, pages * page, _dev(slots), n, None, back, None, heads * D)
                torch.cuda.synchronize()
            found.append((out, lse, kept_idx, mass_out, moved, back))
        for a, b in zip(*found):
            assert torch.equal(a, b)
        assert found[0][0].any()
        del cache, found


def test_cache_copies_and_a_long_eviction_replayed_from_a_graph():
    _say("graph: rows into the cache, a long eviction, rows out of it")
    rng = np.random.default_rng(31)
    heads, D, page, lengths, budget = 4, 64, 64, [25000, 700, 0], 7000
    R, most, row = len(lengths), max(lengths), up.uniprefill_q4_row_bytes(heads, D)
    kept = [min(n, budget) for n in lengths]
    need, new = [-(-n // page) for n in lengths], [-(-n // page) for n in kept]
    table, new_table = np.full((R, max(need)), -1, np.int32), np.full((R, max(new)), -1, np.int32)
    pages, at = rng.permutation(sum(need) + sum(new)), 0
    for t, counts in ((table, need), (new_table, new)):
        for r, n in enumerate(counts):
            t[r, :n] = pages[at:at + n]
            at += n
    slots = np.concatenate([ao.page_rows(table[r], n, page) for r, n in enumerate(lengths)])
    out_slots = np.concatenate([ao.page_rows(new_table[r], n, page) for r, n in enumerate(kept)])
    p = up.make_params(num_seqs=R, total_tokens=sum(lengths), block_size=64, num_q_heads=heads, num_kv_heads=heads, head_dim=D)
    n, m = len(slots), len(out_slots)
    k = torch.zeros(n, heads, D, dtype=BF, device="cuda")
    cache = torch.zeros(at * page, row, dtype=torch.uint8, device="cuda")
    mass = torch.zeros(R, most, device="cuda")
    kept_idx, mass_out = torch.zeros(R, budget, dtype=torch.int32, device="cuda"), torch.zeros(R, budget, device="cuda")
    new_len, back = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(m, heads, D, dtype=BF, device="cuda")
    lens, tab, new_tab, s_in, s_out = (_dev(np.asarray(a)) for a in (np.array(lengths, np.int32), table, new_table, slots, out_slots))

    def calls():
        up.uniprefill_cache_store_q4(p, k, None, heads * D, s_in, n, None, cache, None, row, at * page)
        up.uniprefill_cache_evict(cache, None, row, row, mass, most, lens, R, most, budget, 5, 64, tab, table.shape[1], new_tab,
                                  new_table.shape[1], page, kept_idx, mass_out, budget, new_len)
        up.uniprefill_cache_load_q4(p, cache, None, row, at * page, s_out, m, None, back, None, heads * D)

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(4):
        rows, rows64 = _rows(rng, BF, n, heads, D)
        masses = rng.random((R, most)).astype(np.float32)
        k.copy_(rows)
        mass.copy_(torch.from_numpy(masses))
        back.zero_()
        graph.replay()
        torch.cuda.synchronize()
        a = b = 0
        for r, length in enumerate(lengths):
            stay = ao.evict_tokens(masses[r], length, budget, 5, 64)
            np.testing.assert_array_equal(kept_idx[r, :len(stay)].cpu().numpy(), stay)
            np.testing.assert_array_equal(mass_out[r, :len(stay)].cpu().numpy(), masses[r][stay])
            want = ao.q4_values(*ao.q4_quantise(rows[a:a + length].float().numpy()[stay])) if length else np.zeros((0, heads, D))
            got = back[b:b + len(stay)].double().cpu().numpy()
            assert (np.abs(got - want) <= (2.0 ** -8 + F) * np.abs(want)).all()      # to float, then to bf16
            a, b = a + length, b + len(stay)
        first = [t.clone() for t in (kept_idx, mass_out, new_len, back)]
        calls()
        torch.cuda.synchronize()
        for x, y in zip(first, (kept_idx, mass_out, new_len, back)):
            assert torch.equal(x, y)


def test_prompt_drop_cache_decode_evict_decode():
    """A layer's attention hands its log-sum-exp to the drop; the kept tokens' keys and values enter the 4-bit cache;
    three decode steps read it and accumulate weights; the cache shrinks and decoding goes on."""
    _say("a prompt through attention, drop, cache, decode, eviction, decode")
    hq, hkv, D, page, lengths = 8, 2, 128, 16, [700, 333]
    b = Batch(21, lengths, hq, hkv, D)
    b.run()
    b.check()
    R, T, cu = len(lengths), sum(lengths), b.cu_host
    ratio = np.array([0.3, 0.5], np.float32)
    p = up.make_params(num_seqs=R, total_tokens=T, block_size=64, n_obs=32, n_sink=16, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                       hidden_dim=hkv * D)
    _, new_cu_host, kept, ws_bytes = up.uniprefill_plan(p, cu, ratio)
    ws = torch.empty(ws_bytes + 256, dtype=torch.uint8, device="cuda")
    keys = torch.zeros(kept, hkv * D, dtype=BF, device="cuda")
    vals = torch.zeros_like(keys)
    idx = torch.zeros(kept, dtype=torch.int32, device="cuda")
    new_cu = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    up.uniprefill_fused_lse(p, b.q, b.k, b.lse, b.lse.shape[1], b.k, None, b.cu, cu, None, None, None, 0, page, _dev(ratio), ratio, keys,
                            None, idx, new_cu, None, ws, ws_bytes)
    up.uniprefill_compact(p, b.v, None, idx, kept, vals, None)
    want_kept = oracle.sparsify(b.q64, b.k64, host_bits(b.k), np.arange(T, dtype=np.int32), cu, ratio, block_size=64, n_obs=32,
                                n_sink=16)["kept_idx"]
    np.testing.assert_array_equal(idx.cpu().numpy(), want_kept)
    # the kept tokens take the first slots of their sequences' pages
    room = int(max(np.diff(new_cu_host))) + 8
    per = -(-room // page)
    rng = np.random.default_rng(2)
    pages = rng.permutation(3 * R * per)
    table, new_table = pages[:R * per].reshape(R, per).astype(np.int32), pages[R * per:2 * R * per].reshape(R, per).astype(np.int32)
    stride = up.uniprefill_q4_row_bytes(hkv, D)
    slots_n = len(pages) * page
    kc, vc = (torch.zeros(slots_n, stride, dtype=torch.uint8, device="cuda") for _ in range(2))
    pos = torch.cat([torch.arange(n, dtype=torch.int32) for n in np.diff(new_cu_host)]).cuda()
    slots = torch.zeros(kept, dtype=torch.int64, device="cuda")
    up.uniprefill_slot_mapping(pos, new_cu, R, _dev(table), per, page, kept, slots)
    up.uniprefill_cache_store_q4(p, keys, vals, hkv * D, slots, kept, new_cu[R:], kc, vc, stride, slots_n)
    K, V = b.k64[want_kept].astype(np.float32), b.v64[want_kept].astype(np.float32)
    model = [[ao.q4_pack(*ao.q4_quantise(x[new_cu_host[r]:new_cu_host[r + 1]])) for r in range(R)] for x in (K, V)]
    lens = np.diff(new_cu_host).astype(np.int32)
    mass = torch.zeros(R, room, device="cuda")
    mass64 = [np.zeros(room) for _ in range(R)]
    dp = up.make_params(num_seqs=R, total_tokens=R, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D)
    _, dws_bytes = up.uniprefill_attention_q4_plan(dp, room, True)
    dws = torch.empty(dws_bytes + 256, dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(R, hq, D, dtype=BF, device="cuda"), torch.zeros(hq, R, device="cuda")

    def step(table, mass):
        # the new token's key and value enter, then its query reads them all
        (k1, _), (v1, _), (q1, q64) = _rows(rng, BF, R, hkv, D), _rows(rng, BF, R, hkv, D), _rows(rng, BF, R, hq, D)
        one = torch.zeros(R, dtype=torch.int64, device="cuda")
        up.uniprefill_slot_mapping(_dev(lens), _dev(np.arange(R + 1, dtype=np.int32)), R, _dev(table), per, page, R, one)
        up.uniprefill_cache_store_q4(dp, k1.cuda(), v1.cuda(), hkv * D, one, R, None, kc, vc, stride, slots_n)
        for r in range(R):
            for m, x in zip(model, (k1, v1)):
                m[r] = np.concatenate([m[r], ao.q4_pack(*ao.q4_quantise(x[r:r + 1].float().numpy()))])
        lens[:] += 1
        up.uniprefill_attention_q4(dp, q1.cuda(), kc, vc, stride, _dev(lens), room, _dev(table), per, page, out, hq * D, lse, R, mass,
                                   mass, room, dws, dws_bytes)
        torch.cuda.synchronize()
        for r in range(R):
            want, want_lse, mean, _, near, far, top = ao.decode_attention_q4(q64[r], model[0][r], model[1][r], hkv)
            d = _logit_error(top, D)[:, None]
            tol = 2.0 ** -8 * (np.abs(want) + near) + (2 * d + (lens[r] + 64) * F) * far
            assert (np.abs(out[r].double().cpu().numpy() - want) <= tol).all()
            mass64[r][:lens[r]] += mean
            np.testing.assert_allclose(mass[r].double().cpu().numpy(), mass64[r], rtol=1e-4, atol=1e-12)

    for _ in range(3):
        step(table, mass)
    budget = 150
    kept_idx = torch.zeros(R, budget, dtype=torch.int32, device="cuda")
    mass2 = torch.zeros(R, room, device="cuda")
    new_len = torch.zeros(R, dtype=torch.int32, device="cuda")
    old_mass = mass.cpu().numpy()
    kept_idx = torch.zeros(R, room, dtype=torch.int32, device="cuda")
    up.uniprefill_cache_evict(kc, vc, stride, stride, mass, room, _dev(lens), R, room, budget, 16, 32, _dev(table), per, _dev(new_table), per,
                              page, kept_idx, mass2, room, new_len)
    torch.cuda.synchronize()
    for r in range(R):
        stay = ao.evict_tokens(old_mass[r], int(lens[r]), budget, 16, 32)
        np.testing.assert_array_equal(kept_idx[r, :len(stay)].cpu().numpy(), stay)
        for m in model:
            m[r] = m[r][stay]
        kept_mass = mass64[r][stay]
        mass64[r][:] = 0
        mass64[r][:len(stay)] = kept_mass
        lens[r] = len(stay)
    np.testing.assert_array_equal(new_len.cpu().numpy(), lens)
    for _ in range(2):
        step(new_table, mass2)
