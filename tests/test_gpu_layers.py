"""GPU tests of the operators of the layers between two drops against the 64-bit oracle: windowed attention, linear
attention, norm and rotation, pages for new tokens, and all of them in a row.

Tolerances (F = 2^-24, half a step of float; u = 2^-8 for bf16 results, F for float ones).
  windowed attention: as for uniprefill_attention (tests/test_gpu_attention.py).
  linear attention: with A the same sum over absolute values, a state's element is off by at most (3 n + 512) F A: its
    terms are scaled and added at most three roundings a token each, and an exponential of at most 2^7 in the exponent is
    good to 2^8 F; an output by its own rounding and ((3 n + D + 512) F) A, and for bf16 operands 2^-15 A more (the
    decayed logits and the state in two parts of bf16: 2^-16 each).
  norm and rotation: with B = |a| + |b| of the pair, (D + 40) F B and the result's rounding: D products are added up, and a root, a
    quotient, two weights, a sine and a cosine (4 F each) and four operations follow.  Values that are copied: bit for bit.
  pages: whole numbers, equal."""
import numpy as np
import pytest
import torch

import paper_2605_06221_amd as up
from oracle import attention_oracle as ao
from oracle import layers_oracle as lo
from test_gpu_attention import BF, F, F32, Batch, _attention_tolerance, _cu, _dev, _graph, _lse_tolerance, _rows, _say, _strided

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Window(Batch):
    """A packed batch with everything that a call of uniprefill_attention_window takes.  Pages whose keys no token sees are
    replaced by one that holds NaN."""

    def __init__(self, window, n_sink, *args, **kw):
        super().__init__(*args, **kw)
        self.window, self.n_sink = window, n_sink
        if self.table is not None:
            table = self.table.cpu().numpy()
            gone = int(np.setdiff1d(np.arange(self.k.shape[0] // self.page), table)[0])      # a page of nobody's (NaN)
            for r, (n, m) in enumerate(zip(self.lengths, self.keys)):
                seen = lo.visible(m - n, n, m, window, n_sink).any(axis=0)
                for j in range(-(-m // self.page)):
                    if not seen[j * self.page:(j + 1) * self.page].any():
                        table[r, j] = gone
            self.table = _dev(table)
        _, self.ws_bytes = up.uniprefill_attention_window_plan(self.p, self.cu_host, self.ck_host if self.ctx else None, window, n_sink)
        self.ws = torch.full((self.ws_bytes + 256,), 255, dtype=torch.uint8, device="cuda")

    def run(self, want_lse=True, stream=None):
        return up.uniprefill_attention_window(
            self.p, self.q, self.k, self.v, self.v.shape[1], self.cu, self.cu_host, self.ck if self.ctx else None,
            self.ck_host if self.ctx else None, self.table, self.tstride, max(self.page, 1), self.window, self.n_sink, self.out,
            self.out.shape[1], self.lse if want_lse else None, self.lse.shape[1], self.ws, self.ws_bytes, stream=stream)

    def oracle(self):
        return lo.window_attention(self.q64, self.k64, self.v64, self.cu_host, self.ck_host, self.window, self.n_sink,
                                   scale=self.scale or None, gather=self.gather)

    def check(self, want_lse=True):
        T, hq = int(self.cu_host[-1]), self.lse.shape[0]
        want, lse, absv, top = self.oracle()
        got, got_lse = self.results()
        n = max(self.keys + [1])
        tol = _attention_tolerance(want, absv, top, n, self.D, self.dtype == BF)
        worst = np.max(np.abs(got - want) / tol) if T else 0.0
        _say("  worst error / tolerance", float(worst))
        assert worst <= 1.0, np.unravel_index(np.argmax(np.abs(got - want) / tol), got.shape)
        if want_lse:
            seen = np.isfinite(lse)
            np.testing.assert_array_equal(np.isfinite(got_lse), seen)
            assert (np.abs(got_lse[seen] - lse[seen]) <= _lse_tolerance(lse, top, n, self.D)[seen]).all()
            assert (got_lse[~seen] == -np.inf).all()
        else:
            assert (self.lse == -7.0).all()
        assert (self.out[T:] == -7.0).all() and (self.out[:, hq * self.D:] == -7.0).all() and (self.lse[:, T:] == -7.0).all()


BANDS = [(1, 0), (1, 1), (7, 0), (64, 4), (65, 63), (100, 128), (129, 1), (500, 64), (100000, 5), (2 ** 31 - 1, 2 ** 31 - 1)]


@pytest.mark.parametrize("window,n_sink", BANDS)
@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (64, F32), (128, F32)])
def test_window_attention_of_whole_prompts(window, n_sink, D, dtype):
    _say("window attention", window, n_sink, D, dtype)
    b = Window(window, n_sink, window % 97 + D, [130, 1, 0, 515, 63], 8, 2, D, dtype)
    b.run()
    b.check()


@pytest.mark.parametrize("page", [0, 1, 7, 16, 48])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (33, 4), (250, 70), (640, 0), (5000, 3)])
@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (128, F32)])
def test_window_attention_after_earlier_context(page, window, n_sink, D, dtype):
    _say("window attention after context", page, window, n_sink, D, dtype)
    b = Window(window, n_sink, page + D, [5, 1, 0, 140, 33, 300], 8, 2, D, dtype, earlier=[700, 1300, 9, 0, 61, 450], page=page, pad=16)
    b.run()
    b.check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 1), (64, 1), (6, 2), (40, 8)])
def test_window_attention_head_layouts(hq, hkv):
    _say("window attention, heads", hq, hkv)
    for window, n_sink in ((50, 3), (200, 0)):
        b = Window(window, n_sink, hq, [333, 2, 70], hq, hkv, 64, earlier=[0, 400, 90], page=16)
        b.run()
        b.check()


@pytest.mark.parametrize("lengths,earlier,hq,hkv,D,dtype,window,n_sink", [
    ([1], [20000], 8, 1, 128, BF, 15000, 4), ([1, 1, 3], [5000, 1, 9000], 4, 4, 64, BF, 4000, 100), ([40, 1], [4000, 2500], 8, 2, 256, BF, 3000, 0),
    ([2], [6000], 64, 1, 128, BF, 5001, 65), ([1, 30], [3000, 2100], 5, 5, 128, F32, 1500, 7), ([1] * 300 + [2], [3] * 300 + [9000], 4, 4, 64, BF, 8000, 1),
])
def test_window_attention_with_the_keys_cut_into_pieces(lengths, earlier, hq, hkv, D, dtype, window, n_sink):
    _say("window attention in pieces", lengths[:4], earlier[:4], hq, hkv, D, dtype, window, n_sink)
    for page in (0, 16):
        b = Window(window, n_sink, 7, lengths, hq, hkv, D, dtype, earlier=earlier, page=page)
        assert b.ws_bytes > 0
        b.run()
        b.check()


@pytest.mark.parametrize("lengths,earlier,hq,hkv,D,dtype,page,window,n_sink", [
    ([2100, 1, 67], None, 32, 8, 128, BF, 0, 700, 4), ([1100], [333], 64, 8, 64, BF, 16, 150, 128), ([700, 0, 400], [50, 0, 0], 64, 8, 256, BF, 8, 99, 33),
    ([1010], [129], 64, 16, 128, F32, 24, 400, 1), ([520, 1, 67], None, 256, 16, 64, BF, 0, 64, 0), ([2100, 1], [0, 9000], 32, 8, 128, BF, 16, 1000, 16),
    ([300], [700], 512, 8, 128, BF, 16, 600, 200), ([515], None, 256, 16, 64, F32, 7, 300, 0),
    # windows wide enough for 256 rows whatever the width of the heads
    ([1100], [3000], 64, 8, 64, BF, 16, 2500, 70), ([1100, 40], [2900, 0], 64, 8, 128, BF, 0, 2300, 200), ([1040], [2600], 64, 8, 64, F32, 7, 2100, 1),
    ([1100], [2600], 64, 8, 128, BF, 24, 2222, 0),
])
def test_window_attention_in_work_groups_of_256_rows(lengths, earlier, hq, hkv, D, dtype, page, window, n_sink):
    _say("window attention, large", lengths, earlier, hq, hkv, D, dtype, page, window, n_sink)
    b = Window(window, n_sink, 31, lengths, hq, hkv, D, dtype, earlier=earlier or [0] * len(lengths), page=page)
    b.run()
    b.check()


def test_window_attention_that_sees_everything_equals_attention():
    _say("window attention, window beyond the keys")
    kw = dict(earlier=[900, 0, 20], page=16)
    a, b = Batch(3, [100, 400, 1], 8, 2, 128, **kw), Window(1000, 0, 3, [100, 400, 1], 8, 2, 128, **kw)
    a.run()
    b.run()
    got, want = b.results(), a.results()
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def test_window_attention_strides_scale_no_lse_and_streams():
    _say("window attention: padded rows, scale, no log-sum-exp, another stream, again")
    b = Window(40, 2, 3, [100, 37], 8, 2, 128, pad=24, scale=0.3)
    b.run(want_lse=False)
    b.check(want_lse=False)
    first = b.results()[0]
    b.out.fill_(-7.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.run(want_lse=False, stream=side)
    np.testing.assert_array_equal(first, b.results()[0])


class Step(Window):
    """One new token per sequence at the end of a paged cache."""

    def __init__(self, window, n_sink, seed, lengths, hq, hkv, D, dtype=BF, page=16, pad=0, most=None, slack=0):
        Batch.__init__(self, seed, [1] * len(lengths), hq, hkv, D, dtype, earlier=[max(0, n - 1) for n in lengths], page=page, pad=pad)
        self.window, self.n_sink, self.real = window, n_sink, lengths
        self.keys = [max(0, n) for n in lengths]
        table = self.table.cpu().numpy()
        gone = int(np.setdiff1d(np.arange(self.k.shape[0] // page), table)[0])
        for r, m in enumerate(self.keys):
            seen = lo.visible(m - 1, 1, m, window, n_sink)[0] if m else np.zeros(0, bool)
            for j in range(table.shape[1]):
                if not seen[j * page:(j + 1) * page].any():
                    table[r, j] = gone
        self.table = _dev(table)
        self.ck_host = _cu(self.keys)
        self.max_len = max(self.keys) + slack
        if slack:
            wide = np.full((len(lengths), -(-self.max_len // page)), gone, np.int32)
            wide[:, :table.shape[1]] = table[:, :wide.shape[1]]
            self.table, self.tstride = _dev(wide), wide.shape[1]
        self.kv_len = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        _, self.ws_bytes = up.uniprefill_attention_window_step_plan(self.p, self.max_len, window, n_sink)
        self.ws = torch.full((self.ws_bytes + 256,), 255, dtype=torch.uint8, device="cuda")

    def run(self, want_lse=True, stream=None):
        return up.uniprefill_attention_window_step(
            self.p, self.q, self.k, self.v, self.v.shape[1], self.kv_len, self.max_len, self.table, self.tstride, self.page, self.window,
            self.n_sink, self.out, self.out.shape[1], self.lse if want_lse else None, self.lse.shape[1], self.ws, self.ws_bytes,
            stream=stream)


STEP_LENGTHS = [700, 1, 0, 63, 64, 65, 1300, 129, 2000]


@pytest.mark.parametrize("window,n_sink", BANDS)
@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (64, F32), (128, F32)])
def test_step_of_ragged_caches(window, n_sink, D, dtype):
    _say("step", window, n_sink, D, dtype)
    b = Step(window, n_sink, window % 89 + D, STEP_LENGTHS, 8, 2, D, dtype)
    b.run()
    b.check()


@pytest.mark.parametrize("page", [1, 7, 16, 48, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 1), (64, 1), (34, 2), (40, 8), (8, 8)])
def test_step_pages_and_head_layouts(page, hq, hkv):
    _say("step, page", page, "heads", hq, hkv)
    for D, dtype, window, n_sink in ((128, BF, 300, 4), (64, F32, 900, 33)):
        b = Step(window, n_sink, page, STEP_LENGTHS, hq, hkv, D, dtype, page=page, pad=8, slack=100)
        b.run()
        b.check()


@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (128, F32)])
def test_step_with_long_windows(D, dtype):
    _say("step, long", D, dtype)
    for lengths, window, n_sink in (([9000], 8500, 4), ([9000, 30, 7000], 5000, 200), ([12000], 2 ** 31 - 1, 0)):
        b = Step(window, n_sink, D, lengths, 8, 2, D, dtype)
        b.run()
        b.check()


def test_step_lengths_are_clamped_and_read_from_replay_to_replay():
    _say("step: lengths out of range, a captured call")
    b = Step(100, 4, 5, [400, 77, 1], 8, 2, 128, slack=0)
    g = _graph(b.run)
    for lengths in ([400, 77, 1], [399, 0, 1], [400, -5, 2 ** 31 - 1], [150, 30, 0]):
        real = [max(0, min(400, n)) for n in lengths]
        if real[2] > 1:
            b.kv_len.copy_(torch.tensor([lengths[2], lengths[1], 1], dtype=torch.int32))
            real = [real[2], real[1], 1]
        else:
            b.kv_len.copy_(torch.tensor(lengths, dtype=torch.int32))
        # (the windows reach back to what a shorter sequence sees: the whole table again)
        whole = Batch(5, [1, 1, 1], 8, 2, 128, earlier=[399, 76, 0], page=16)
        b.table.copy_(whole.table)
        b.keys, b.ck_host = real, _cu(real)
        b.out.fill_(-7.0)
        b.lse.fill_(-7.0)
        g.replay()
        b.check()


# ---------------------------------------------------------------------------------------------------- linear attention
class Linear:
    def __init__(self, seed, lengths, hq, hkv, D, dtype=BF, log_decay=None, starts=None, stores=None, pad=0, scale=0.0, step=False):
        rng = np.random.default_rng(seed)
        self.lengths, self.D, self.dtype, self.hq, self.hkv, self.scale, self.step = lengths, D, dtype, hq, hkv, scale, step
        n_seqs, T = len(lengths), sum(lengths)
        self.cu_host = _cu(lengths)
        q, self.q64 = _rows(rng, dtype, T, hq, D)
        k, self.k64 = _rows(rng, dtype, T, hkv, D)
        v, self.v64 = _rows(rng, dtype, T, hkv, D)
        self.q, self.k, self.v = (_strided(torch.cat([t, torch.full((1, *t.shape[1:]), NAN, dtype=dtype)]), pad, NAN) for t in (q, k, v))
        self.ld = np.asarray(-2.0 ** (-8.0 * np.arange(1, hkv + 1) / hkv) if log_decay is None else np.resize(log_decay, hkv), np.float32)
        self.log_decay, self.cu = _dev(self.ld), _dev(self.cu_host)
        self.num, self.stride = n_seqs + 2, hkv * D * D + 4 * pad
        pool = torch.full((self.num, self.stride), NAN)
        self.start = rng.standard_normal((self.num, hkv, D, D)).astype(np.float32)
        pool[:, :hkv * D * D] = torch.from_numpy(self.start.reshape(self.num, -1))
        self.pool0 = pool
        self.pool = pool.cuda()
        self.state_in = None if starts is None else np.asarray(starts, np.int32)
        self.state_out = None if stores is None else np.asarray(stores, np.int32)
        self.out = torch.full((T + 3, hq * D + pad), -7.0, dtype=dtype, device="cuda")
        self.p = up.make_params(num_seqs=n_seqs, total_tokens=T, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                                q_row_stride=hq * D + pad, k_row_stride=hkv * D + pad, softmax_scale=scale,
                                qk_dtype=up.UP_F32 if dtype == F32 else up.UP_BF16)
        self.in_dev = None if starts is None else _dev(self.state_in)
        self.out_dev = None if stores is None else _dev(self.state_out)
        if not step:
            _, self.ws_bytes = up.uniprefill_linear_attention_plan(self.p, self.cu_host)
            self.ws = torch.full((self.ws_bytes + 256,), 255, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        states = [self.log_decay, self.pool, self.stride, self.num, self.in_dev, self.out_dev]
        if self.step:
            return up.uniprefill_linear_attention_step(self.p, self.q, self.k, self.v, self.v.shape[1], *states, self.out, self.out.shape[1],
                                                       stream=stream)
        return up.uniprefill_linear_attention(self.p, self.q, self.k, self.v, self.v.shape[1], self.cu, self.cu_host, *states, self.out,
                                              self.out.shape[1], self.ws, self.ws_bytes, stream=stream)

    def results(self):
        torch.cuda.synchronize()
        T = int(self.cu_host[-1])
        pool = self.pool[:, :self.hkv * self.D * self.D].double().cpu().numpy().reshape(self.num, self.hkv, self.D, self.D)
        return self.out[:T, :self.hq * self.D].double().cpu().numpy().reshape(T, self.hq, self.D), pool

    def check(self):
        T, n = int(self.cu_host[-1]), max(self.lengths + [1])
        want, pool, bound, pool_bound = lo.linear_attention(self.q64, self.k64, self.v64, self.cu_host, self.ld, self.start, self.state_in,
                                                            self.state_out, scale=self.scale or None)
        got, got_pool = self.results()
        u = 2.0 ** -8 if self.dtype == BF else F
        tol = u * np.abs(want) + ((3 * n + self.D + 512) * F + (2.0 ** -15 if self.dtype == BF else 0.0)) * bound + 1e-30
        ptol = (3 * n + 512) * F * pool_bound
        worst = np.max(np.abs(got - want) / tol) if T else 0.0
        with np.errstate(divide="ignore", invalid="ignore"):
            off = np.abs(got_pool - pool)
            pworst = np.max(np.where(off == 0, 0.0, off / ptol))      # (slots that nobody stores to: the same bits)
        _say("  worst error / tolerance", float(worst), "states", float(pworst))
        assert worst <= 1.0, np.unravel_index(np.argmax(np.abs(got - want) / tol), got.shape)
        assert pworst <= 1.0, np.unravel_index(np.argmax(np.where(off == 0, 0.0, off / ptol)), off.shape)
        assert (self.out[T:] == -7.0).all() and (self.out[:, self.hq * self.D:] == -7.0).all()
        assert torch.isnan(self.pool[:, self.hkv * self.D * self.D:]).all()


def _slots(n, *, fresh=3, none=4):
    """Slots that n sequences start from and store to: some from zero, some not stored, one named by a number past the pool."""
    starts = [(-1 if i % fresh == 0 else i + 1) for i in range(n)]
    stores = [(n + 2 if i % none == 3 else i + 1) for i in range(n)]
    return starts, stores


TYPES = [(64, BF), (128, BF), (256, BF), (64, F32), (128, F32)]


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("lengths,hq,hkv", [([1], 1, 1), ([1, 0, 2, 31, 32, 33], 8, 2), ([129, 0, 1, 65], 5, 1), ([64, 63], 6, 6), ([200], 64, 1)])
def test_linear_attention(lengths, hq, hkv, D, dtype):
    _say("linear attention", lengths, hq, hkv, D, dtype)
    starts, stores = _slots(len(lengths))
    b = Linear(len(lengths) + D, lengths, hq, hkv, D, dtype, starts=starts, stores=stores)
    b.run()
    b.check()


@pytest.mark.parametrize("D,dtype", [(64, BF), (128, BF), (256, BF), (128, F32)])
@pytest.mark.parametrize("decay", [[0.0], [-1e-4], [-0.02], [-1.0], [-30.0], [-1e30], [-float("inf")], [0.7, -3.0]])
def test_linear_attention_decays(decay, D, dtype):
    # none at all, slow and fast ones, some that leave nothing after one token, one above 0 (counts as 0)
    _say("linear attention, log decay", decay, D, dtype)
    b = Linear(17, [700, 90], 4, 2, D, dtype, log_decay=decay, starts=[0, -1], stores=[0, 1], pad=8)
    b.run()
    b.check()


@pytest.mark.parametrize("D,dtype", TYPES)
def test_linear_attention_of_long_sequences(D, dtype):
    _say("linear attention, long", D, dtype)
    b = Linear(23, [3000, 1, 2049], 2, 1, D, dtype, log_decay=[-0.003], starts=[2, 3, -1], stores=[2, 3, 0])
    b.run()
    b.check()


@pytest.mark.parametrize("D,dtype", [(64, BF), (256, BF), (128, F32)])
def test_linear_attention_at_the_borders_of_pieces(D, dtype):
    # pieces of 64 tokens: one, two, eight, nine and seventeen whole ones, and a token more or less
    lengths = [64, 65, 128, 512, 513, 576, 577, 1088, 1087]
    _say("linear attention, whole pieces", D, dtype)
    starts, stores = _slots(len(lengths))
    b = Linear(29, lengths, 2, 1, D, dtype, log_decay=[-0.01], starts=starts, stores=stores)
    b.run()
    b.check()


def test_linear_attention_without_states_with_a_scale_and_in_two_calls():
    _say("linear attention: no pool, scale; one call against two")
    b = Linear(5, [150, 40], 4, 2, 128, scale=1.0)
    b.run()
    b.check()
    whole = Linear(6, [300], 4, 4, 128, starts=[-1], stores=[1])
    first, second = Linear(6, [170], 4, 4, 128, starts=[-1], stores=[1]), Linear(6, [130], 4, 4, 128, starts=[1], stores=[1])
    for name in ("q", "k", "v"):
        rows = getattr(whole, name)
        getattr(first, name)[:170] = rows[:170]
        getattr(second, name)[:130] = rows[170:300]
    whole.run()
    first.run()
    second.pool = first.pool
    second.run()
    want, want_pool = whole.results()
    got, got_pool = second.results()
    np.testing.assert_allclose(got, want[170:], rtol=2.0 ** -6, atol=0.02)      # (two bf16 roundings of sums that differ in float)
    np.testing.assert_allclose(got_pool[1], want_pool[1], rtol=1e-4, atol=1e-4)
    whole.check()


def test_linear_attention_runs_streams_and_replays():
    _say("linear attention: the same on every run, another stream, a captured call with new rows")
    starts, stores = _slots(4)
    b = Linear(8, [1100, 0, 65, 1], 8, 2, 128, starts=starts, stores=stores)
    b.run()
    first = b.results()
    side = torch.cuda.Stream()
    for i in range(4):
        b.out.fill_(-7.0)
        b.ws.fill_(i)
        b.pool.copy_(b.pool0)
        torch.cuda.synchronize()
        b.run(stream=side if i % 2 else None)
        for x, y in zip(first, b.results()):
            np.testing.assert_array_equal(x, y)
    g = _graph(b.run)
    rng = np.random.default_rng(3)
    for i in range(3):
        q, b.q64 = _rows(rng, BF, *b.q64.shape)
        b.q[:-1] = q.reshape(q.shape[0], -1).cuda()
        b.out.fill_(-7.0)
        b.pool.copy_(b.pool0)
        g.replay()
        b.check()


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 2), (64, 1), (3, 3), (40, 8)])
def test_linear_attention_step(hq, hkv, D, dtype):
    _say("linear attention, one token", hq, hkv, D, dtype)
    for n in (1, 7):
        starts, stores = _slots(n)
        b = Linear(n + D, [1] * n, hq, hkv, D, dtype, starts=starts, stores=stores, pad=8, step=True)
        b.run()
        b.check()


def test_linear_attention_steps_follow_the_chunks():
    _say("linear attention: a prompt, then 60 replayed steps, against the whole")
    n, more = 90, 60
    whole = Linear(12, [n + more], 8, 2, 128, starts=[-1], stores=[0])
    head, step = Linear(12, [n], 8, 2, 128, starts=[-1], stores=[0]), Linear(13, [1], 8, 2, 128, starts=[0], stores=[0], step=True)
    for name in ("q", "k", "v"):
        getattr(head, name)[:n] = getattr(whole, name)[:n]
    head.run()
    step.pool.copy_(head.pool)
    keep = step.pool.clone()
    g = _graph(step.run)
    step.pool.copy_(keep)
    whole.run()
    whole.check()
    want, pool = whole.results()
    u = 2.0 ** -8
    for i in range(more):
        for name in ("q", "k", "v"):
            getattr(step, name)[0] = getattr(whole, name)[n + i]
        g.replay()
        got = step.results()[0][0]
        np.testing.assert_allclose(got, want[n + i], rtol=2 * u, atol=2e-3)      # (the roundings of both, and the chunk's 16 bits)
    np.testing.assert_allclose(step.results()[1][0], pool[0], rtol=1e-4, atol=1e-4)


# ---------------------------------------------------------------------------------------------------- norm and rotation
class Rotate:
    def __init__(self, seed, tokens, hq, hkv, D, dtype=BF, rot=None, pairs=False, norm=True, weights=True, slots=True, pos=None, pad=0):
        rng = np.random.default_rng(seed)
        self.n, self.hq, self.hkv, self.D, self.dtype, self.pairs, self.pad = tokens, hq, hkv, D, dtype, pairs, pad
        self.rot, self.eps = D if rot is None else rot, 1e-5 if norm else 0.0
        self.row = (hq + 2 * hkv) * D + pad
        x, self.x64 = _rows(rng, dtype, tokens, hq + 2 * hkv, D)
        self.x = _strided(x, pad, NAN)
        w, self.w64 = _rows(rng, dtype, 2, D)
        self.weights = norm and weights
        self.w = w.cuda() if self.weights else None
        self.pos_host = np.asarray(rng.integers(0, 200000, tokens) if pos is None else pos, np.int32)
        self.pos = _dev(self.pos_host)
        self.freq_host = (10000.0 ** (-np.arange(0, self.rot, 2) / max(1, self.rot))).astype(np.float32)
        self.freq = _dev(self.freq_host)
        self.num = tokens + 9
        self.slot_host = rng.permutation(self.num)[:tokens].astype(np.int64)
        if slots and tokens > 4:
            self.slot_host[1], self.slot_host[3] = -1, self.num      # padding
        self.slots = _dev(self.slot_host) if slots else None
        rows = self.num if slots else tokens
        self.q_out = torch.full((tokens + 2, hq * D + pad), -7.0, dtype=dtype, device="cuda")
        self.k_out = torch.full((rows + 1, hkv * D + 2 * pad), -7.0, dtype=dtype, device="cuda")
        self.v_out = torch.full((rows + 1, hkv * D + pad), -7.0, dtype=dtype, device="cuda")
        self.p = up.make_params(num_seqs=1, total_tokens=tokens, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                                q_row_stride=self.row, k_row_stride=self.row, qk_dtype=up.UP_F32 if dtype == F32 else up.UP_BF16)

    def views(self):
        a, b, D = self.hq * self.D, (self.hq + self.hkv) * self.D, self.D
        return self.x[:, :a], self.x[:, a:b], self.x[:, b:b + self.hkv * D]

    def run(self, count=None, stream=None, want=(True, True, True)):
        q, k, v = (t if w else None for t, w in zip(self.views(), want))
        outs = [t if w else None for t, w in zip((self.q_out, self.k_out, self.v_out), want)]
        return up.uniprefill_norm_rotate(self.p, q, k, v, self.row, self.w[0] if self.weights else None, self.w[1] if self.weights else None,
                                         self.eps, self.pos, self.freq, self.rot, self.pairs, count, outs[0], self.q_out.shape[1], outs[1],
                                         self.k_out.shape[1], outs[2], self.v_out.shape[1], self.slots, self.num, stream=stream)

    def check(self, count=None, want=(True, True, True)):
        torch.cuda.synchronize()
        n = self.n if count is None else max(0, min(self.n, count))
        u = 2.0 ** -8 if self.dtype == BF else F
        a, b = self.hq, self.hq + self.hkv
        dst = self.slot_host if self.slots is not None else np.arange(self.n)
        kept = [t for t in range(n) if 0 <= dst[t] < self.num]
        for part, out, rows, there in ((0, self.q_out, np.arange(n), want[0]), (1, self.k_out, dst[kept], want[1])):
            src = self.x64[:n, :a] if part == 0 else self.x64[kept, a:b]
            pos = self.pos_host[:n] if part == 0 else self.pos_host[kept]
            ref, size = lo.norm_rotate(src, self.w64[part] if self.weights else None, self.eps, pos, self.freq_host, self.rot, self.pairs)
            heads = src.shape[1]
            if there:
                got = out[_dev(np.asarray(rows, np.int64)), :heads * self.D].double().cpu().numpy().reshape(ref.shape)
                tol = u * np.abs(ref) + (self.D + 40) * F * size
                if self.eps == 0 and self.rot < self.D:
                    np.testing.assert_array_equal(got[..., self.rot:], src[..., self.rot:])
                assert (np.abs(got - ref) <= tol).all(), np.unravel_index(np.argmax(np.abs(got - ref) - tol), ref.shape)
            left = np.setdiff1d(np.arange(out.shape[0]), rows) if there else np.arange(out.shape[0])
            assert (out[_dev(left)] == -7.0).all() and (out[:, heads * self.D:] == -7.0).all()
        if want[2]:
            got = self.v_out[_dev(np.asarray(dst[kept], np.int64)), :self.hkv * self.D]
            assert torch.equal(got.cpu(), self.views()[2][_dev(np.asarray(kept, np.int64))].cpu())
        left = np.setdiff1d(np.arange(self.v_out.shape[0]), dst[kept]) if want[2] else np.arange(self.v_out.shape[0])
        assert (self.v_out[_dev(left)] == -7.0).all() and (self.v_out[:, self.hkv * self.D:] == -7.0).all()


@pytest.mark.parametrize("D,dtype", TYPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_norm_and_rotation(D, dtype, pairs, norm):
    _say("rotate", D, dtype, "pairs", pairs, "norm", norm)
    for rot in sorted({0, 16, 32, D // 2, D // 2 + 16, D}):
        for tokens, hq, hkv in ((1, 1, 1), (9, 5, 1), (130, 40, 8)):
            b = Rotate(rot + D, tokens, hq, hkv, D, dtype, rot=rot, pairs=pairs, norm=norm, pad=16)
            b.run()
            b.check()


def test_norm_without_weights_and_rows_in_place():
    _say("rotate: no weights; rows of queries and keys where they are")
    b = Rotate(1, 77, 8, 2, 128, weights=False, slots=False)
    b.run()
    b.check()
    c = Rotate(1, 77, 8, 2, 128, weights=False, slots=False)
    q, k, _ = c.views()
    up.uniprefill_norm_rotate(c.p, q, k, None, 0, None, None, c.eps, c.pos, c.freq, c.rot, 0, None, q, c.row, k, c.row, None, 0, None, 0)
    assert torch.equal(c.views()[0], b.q_out[:77]) and torch.equal(c.views()[1], b.k_out[:77])
    assert torch.equal(c.views()[2], b.views()[2])


def test_rotation_of_single_tensors_counts_streams_and_replays():
    _say("rotate: one tensor alone, a count on the device, another stream, a captured call")
    for want in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        b = Rotate(2, 40, 8, 2, 64)
        b.run(want=want)
        b.check(want=want)
    b = Rotate(3, 50, 8, 2, 128)
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = _graph(lambda: b.run(count=count))
    for n in (0, 17, 50, 2 ** 31 - 1, -4):
        count.fill_(n)
        for t in (b.q_out, b.k_out, b.v_out):
            t.fill_(-7.0)
        g.replay()
        b.check(count=n)
    for t in (b.q_out, b.k_out, b.v_out):
        t.fill_(-7.0)
    torch.cuda.synchronize()
    b.run(stream=torch.cuda.Stream())
    b.check()


def test_rotation_at_far_positions_and_of_zero_rows():
    _say("rotate: positions to the ends of their type, rows of zeros")
    pos = [0, 1, 131071, 10 ** 6, 2 ** 31 - 1, -1, -2 ** 31, 5]
    for dtype in (F32, BF):
        b = Rotate(4, 8, 4, 2, 128, dtype, norm=False, pos=pos, slots=False)
        b.run()
        b.check()
    b = Rotate(5, 8, 4, 2, 128, pos=pos)
    b.x.zero_()
    b.x64 = np.zeros_like(b.x64)
    b.run()
    b.check()


def test_rotation_past_the_cache_gives_the_same_bits():
    _say("rotate: more bytes than the cache holds, against the same rows in parts")
    n, hq, hkv, D = 12001, 40, 8, 128
    b = Rotate(6, n, hq, hkv, D)
    assert 2 * n * (hq + 2 * hkv) * D * 2 > 256 << 20
    b.run()
    q, k, v = b.views()
    want_q, want_k, want_v = (torch.full_like(t, -7.0) for t in (b.q_out, b.k_out, b.v_out))
    for lo in range(0, n, 3000):
        hi = min(n, lo + 3000)
        p = up.make_params(num_seqs=1, total_tokens=hi - lo, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, q_row_stride=b.row,
                           k_row_stride=b.row)
        up.uniprefill_norm_rotate(p, q[lo:], k[lo:], v[lo:], b.row, b.w[0], b.w[1], b.eps, b.pos[lo:hi].clone(), b.freq, b.rot, 0, None, want_q[lo:],
                                  hq * D, want_k, hkv * D, want_v, hkv * D, b.slots[lo:hi].clone(), b.num)
    for got, want in ((b.q_out, want_q), (b.k_out, want_k), (b.v_out, want_v)):
        assert torch.equal(got, want)


# ---------------------------------------------------------------------------------------------------- pages
class Pages:
    def __init__(self, seed, lengths, new, page, spare=3, slack=2, capacity=None):
        rng = np.random.default_rng(seed)
        self.n, self.page, self.capacity = len(lengths), page, sum(max(0, x) for x in new) + 5 if capacity is None else capacity
        have = [-(-max(0, n) // page) for n in lengths]
        need = [-(-(max(0, n) + max(0, a)) // page) for n, a in zip(lengths, new)]
        ids = rng.permutation(sum(have) + sum(need) + 50)
        self.table_host = np.full((self.n, max(need + [0]) + slack), -1, np.int32)
        at = 0
        for r, m in enumerate(have):
            self.table_host[r, :m] = ids[at:at + m]
            at += m
        self.free_host = ids[at:].astype(np.int32)
        self.num_free = max(0, min(len(self.free_host), sum(need) - sum(have) + spare))
        self.len_host, self.new_host = np.asarray(lengths, np.int32), np.asarray(new, np.int32)
        self.reset()

    def reset(self):
        self.table, self.free, self.num = _dev(self.table_host), _dev(self.free_host), torch.tensor([self.num_free], dtype=torch.int32, device="cuda")
        self.kv_len, self.new = _dev(self.len_host), _dev(self.new_host)
        full = lambda n, t=torch.int32: torch.full((n,), -77, dtype=t, device="cuda")
        self.new_len, self.left, self.served = full(self.n + 1), full(2), full(2)
        self.cu, self.cu_k, self.pos, self.slots = full(self.n + 2), full(self.n + 2), full(self.capacity + 1), full(self.capacity + 1, torch.int64)

    def run(self, in_place=False, stream=None):
        return up.uniprefill_append_pages(self.kv_len, self.new, self.n, self.page, self.table, self.table_host.shape[1], self.free, self.num,
                                          self.num if in_place else self.left, self.kv_len if in_place else self.new_len, self.cu, self.cu_k,
                                          self.pos, self.slots, self.capacity, self.served, stream=stream)

    def check(self, in_place=False):
        torch.cuda.synchronize()
        want = lo.append_pages(self.len_host, self.new_host, self.page, self.table_host, self.free_host, self.num_free, self.capacity)
        np.testing.assert_array_equal(self.table.cpu().numpy(), want["table"])
        for name, got, n in (("new_len", self.kv_len if in_place else self.new_len, self.n), ("cu", self.cu, self.n + 1),
                             ("cu_k", self.cu_k, self.n + 1), ("pos", self.pos, self.capacity), ("slots", self.slots, self.capacity)):
            np.testing.assert_array_equal(got[:n].cpu().numpy(), np.asarray(want[name]), err_msg=name)
            assert (got[n:] == -77).all()
        assert int((self.num if in_place else self.left)[0]) == want["free_left"] and int(self.served[0]) == want["served"]
        assert (self.served[1:] == -77).all()
        return want


def _requests(seed, n, most):
    rng = np.random.default_rng(seed)
    return [int(x) for x in rng.integers(0, 300, n)], [int(x) for x in rng.choice([0, 1, 1, 17, most], n)]


@pytest.mark.parametrize("page", [1, 7, 16, 128])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1023, 1024, 1025, 2500, 4095, 4096, 4097, 9000])
def test_pages(n, page):
    _say("pages", n, page)
    lengths, new = _requests(n + page, n, 130)
    for spare in (3, 0, -1, -10 ** 6):
        b = Pages(n, lengths, new, page, spare=spare)
        b.run()
        b.check()
    b = Pages(n, lengths, new, page)
    b.run(in_place=True)
    b.check(in_place=True)


def test_pages_limits():
    _say("pages: no sequences, none new, rows and capacity too short, negative numbers, long prompts")
    for lengths, new, kw in (([], [], {}), ([5, 0, 16], [0, 0, 0], {}), ([5, 15, 16, 3], [1, 1, 40, 1], dict(slack=-1)), ([4, 4, 4], [2, 2, 2], dict(capacity=5)),
                             ([4, 4], [2, 2], dict(capacity=0)), ([-3, 16, 40], [5, -2, -7], {}), ([0, 100000, 31], [50000, 70001, 1], {}),
                             ([10, 20], [2 ** 31 - 11, 1], dict(capacity=50, slack=0))):
        if kw.get("slack") == 0:      # a length that the type cannot hold: without the table that it would need
            b = Pages(1, [10, 20], [1, 1], 16)
            b.new_host = np.asarray(new, np.int32)
            b.reset()
        else:
            b = Pages(1, lengths, new, 16, **kw)
        b.run()
        b.check()


def test_pages_step_by_step_in_a_graph():
    _say("pages: a captured step in place, replayed until the pages are used up")
    lengths, new = [14, 0, 33, 16, 5], [1, 1, 1, 1, 1]
    b = Pages(3, lengths, new, 16, spare=6, slack=4, capacity=8)
    b.run(in_place=True)
    b.reset()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        b.run(in_place=True)
    for i in range(60):
        g.replay()
        want = b.check(in_place=True)
        b.len_host, b.num_free, b.table_host = np.asarray(want["new_len"], np.int32), want["free_left"], want["table"].astype(np.int32)
    assert want["served"] < 5


# ---------------------------------------------------------------------------------------------------- all of them in a row
def test_the_layers_of_a_hybrid_model_in_a_row():
    """Two requests, one of them new, the other with cached context: pages for their tokens, norm and rotation into the cache, windowed
    attention over it, linear attention of the same rows from and to states; then a drop of tokens and the layers behind it on what is left;
    then three decode steps, captured once and replayed.  Every stage against the oracle on what the stage before left."""
    _say("pages, rotation, windowed and linear attention, a drop, decode steps")
    rng = np.random.default_rng(77)
    hq, hkv, D, page, window, n_sink = 8, 2, 128, 16, 40, 4
    u = 2.0 ** -8
    had, new = [37, 0], [150, 93]
    R, T, most, pool = 2, sum(new), 20, 64
    table_host = np.full((R, most), -1, np.int32)
    order = rng.permutation(pool).astype(np.int32)
    table_host[0, :3] = order[:3]
    free_host = order[3:]
    table, free = _dev(table_host), _dev(free_host)
    num_free, kv_len = torch.tensor([len(free_host)], dtype=torch.int32, device="cuda"), torch.tensor(had, dtype=torch.int32, device="cuda")
    cu, cu_k, served = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (R + 1, R + 1, 1))
    pos, slots = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    k_cache, _ = _rows(rng, BF, pool * page, hkv, D)
    v_cache, _ = _rows(rng, BF, pool * page, hkv, D)
    k_cache, v_cache = k_cache.cuda().reshape(-1, hkv * D), v_cache.cuda().reshape(-1, hkv * D)
    states = torch.from_numpy(rng.standard_normal((2, hkv, D, D)).astype(np.float32)).cuda()
    ld = np.array([-0.2, -0.01], np.float32)
    log_decay, state_slot = _dev(ld), _dev(np.array([1, 0], np.int32))
    state_from = _dev(np.array([1, -1], np.int32))
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    w, w64 = _rows(rng, BF, 2, D)
    w, freq_dev = w.cuda(), _dev(freq)

    def ints(x):
        return x.cpu().numpy()

    def params(tokens, seqs=R):
        return up.make_params(num_seqs=seqs, total_tokens=tokens, block_size=64, num_q_heads=hq, num_kv_heads=hkv, head_dim=D)

    def host(x, heads):
        return x.double().cpu().numpy().reshape(-1, heads, D)

    # ---- a prompt and a chunk
    want = lo.append_pages(had, new, page, table_host, free_host, len(free_host), T)
    up.uniprefill_append_pages(kv_len, _dev(np.array(new, np.int32)), R, page, table, most, free, num_free, num_free, kv_len, cu, cu_k, pos, slots, T, served)
    for name, got in (("table", table), ("new_len", kv_len), ("cu", cu), ("cu_k", cu_k), ("pos", pos), ("slots", slots)):
        np.testing.assert_array_equal(ints(got), np.asarray(want[name]), err_msg=name)
    q, q64 = _rows(rng, BF, T, hq, D)
    k, k64 = _rows(rng, BF, T, hkv, D)
    v, v64 = _rows(rng, BF, T, hkv, D)
    q, k, v = (t.cuda() for t in (q, k, v))
    q_out = torch.empty_like(q)
    p = params(T)
    up.uniprefill_norm_rotate(p, q, k, v, hkv * D, w[0], w[1], 1e-6, pos, freq_dev, D, 0, None, q_out, hq * D, k_cache, hkv * D, v_cache, hkv * D, slots, pool * page)
    ref, size = lo.norm_rotate(q64, w64[0], 1e-6, want["pos"], freq, D, False)
    assert (np.abs(host(q_out, hq) - ref) <= u * np.abs(ref) + (D + 40) * F * size).all()
    ref, size = lo.norm_rotate(k64, w64[1], 1e-6, want["pos"], freq, D, False)
    assert (np.abs(host(k_cache, hkv)[want["slots"]] - ref) <= u * np.abs(ref) + (D + 40) * F * size).all()
    assert torch.equal(v_cache[slots], v.reshape(T, -1))
    cu_host, ck_host = np.asarray(want["cu"], np.int32), np.asarray(want["cu_k"], np.int32)
    _, nb = up.uniprefill_attention_window_plan(p, cu_host, ck_host, window, n_sink)
    ws = torch.empty(nb + 256, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(hq, T, device="cuda")
    up.uniprefill_attention_window(p, q_out, k_cache, v_cache, hkv * D, cu, cu_host, cu_k, ck_host, table, most, page, window, n_sink, out, hq * D, lse, T, ws, nb)
    gather = lambda r, n: ao.page_rows(want["table"][r].astype(np.int32), n, page)
    o, z, absv, top = lo.window_attention(host(q_out, hq), host(k_cache, hkv), host(v_cache, hkv), cu_host, ck_host, window, n_sink, gather=gather)
    assert (np.abs(host(out, hq) - o) <= _attention_tolerance(o, absv, top, max(want["new_len"]), D, True)).all()
    assert (np.abs(lse.double().cpu().numpy() - z) <= _lse_tolerance(z, top, max(want["new_len"]), D)).all()

    def linear(tokens, q, k, v, cu, cu_host, start):
        before = states.double().cpu().numpy()
        p = params(tokens)
        _, nb = up.uniprefill_linear_attention_plan(p, cu_host)
        ws = torch.empty(nb + 256, dtype=torch.uint8, device="cuda")
        y = torch.empty_like(q)
        up.uniprefill_linear_attention(p, q, k, v, hkv * D, cu, cu_host, log_decay, states, hkv * D * D, 2, start, state_slot, y, hq * D, ws, nb)
        o, pool, bound, pbound = lo.linear_attention(host(q, hq), host(k, hkv), host(v, hkv), cu_host, ld, before, ints(start), ints(state_slot))
        n = int(np.diff(cu_host).max())
        assert (np.abs(host(y, hq) - o) <= u * np.abs(o) + ((3 * n + D + 512) * F + 2.0 ** -15) * bound).all()
        assert (np.abs(states.double().cpu().numpy() - pool) <= (3 * n + 512) * F * pbound).all()
    linear(T, q, k, v, cu, cu_host, state_from)

    # ---- a drop, and the layers behind it on the tokens that stay
    keep = np.sort(rng.permutation(T)[:101]).astype(np.int32)
    kept_cu_host = np.searchsorted(keep, cu_host).astype(np.int32)
    kept, kept_cu, n = _dev(keep), _dev(kept_cu_host), len(keep)
    q2, k2, v2 = (t[kept.long()].contiguous() for t in (q, k, v))
    pos2 = torch.empty(n, dtype=torch.int32, device="cuda")
    up.uniprefill_compact_column(pos, 4, kept, n, None, pos2)
    k2_out, v2_out, q2_out = torch.empty_like(k2), torch.empty_like(v2), torch.empty_like(q2)
    p2 = params(n)
    up.uniprefill_norm_rotate(p2, q2, k2, v2, hkv * D, None, None, 1e-6, pos2, freq_dev, D, 0, None, q2_out, hq * D, k2_out, hkv * D, v2_out, hkv * D, None, 0)
    ref, size = lo.norm_rotate(host(k2, hkv), None, 1e-6, np.asarray(want["pos"])[keep], freq, D, False)
    assert (np.abs(host(k2_out, hkv) - ref) <= u * np.abs(ref) + (D + 40) * F * size).all()
    _, nb = up.uniprefill_attention_window_plan(p2, kept_cu_host, None, window, n_sink)
    ws = torch.empty(nb + 256, dtype=torch.uint8, device="cuda")
    out2 = torch.empty_like(q2)
    up.uniprefill_attention_window(p2, q2_out, k2_out, v2_out, hkv * D, kept_cu, kept_cu_host, None, None, None, 0, page, window, n_sink, out2, hq * D, None, 0, ws, nb)
    o, _, absv, top = lo.window_attention(host(q2_out, hq), host(k2_out, hkv), host(v2_out, hkv), kept_cu_host, kept_cu_host, window, n_sink)
    assert (np.abs(host(out2, hq) - o) <= _attention_tolerance(o, absv, top, n, D, True)).all()
    linear(n, q2, k2, v2, kept_cu, kept_cu_host, state_slot)

    # ---- decode steps of both, from a graph
    p3 = params(R)
    one = torch.ones(R, dtype=torch.int32, device="cuda")
    q3, k3, v3 = (torch.zeros(R, h * D, dtype=BF, device="cuda") for h in (hq, hkv, hkv))
    q3_out, out3, y3 = torch.zeros_like(q3), torch.zeros_like(q3), torch.zeros_like(q3)
    lse3 = torch.zeros(hq, R, device="cuda")
    _, nb3 = up.uniprefill_attention_window_step_plan(p3, most * page, window, n_sink)
    ws3 = torch.empty(nb3 + 256, dtype=torch.uint8, device="cuda")
    pos3, slots3 = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, dtype=torch.int64, device="cuda")

    def step():
        up.uniprefill_append_pages(kv_len, one, R, page, table, most, free, num_free, num_free, kv_len, cu, cu_k, pos3, slots3, R, served)
        up.uniprefill_norm_rotate(p3, q3, k3, v3, hkv * D, w[0], w[1], 1e-6, pos3, freq_dev, D, 0, None, q3_out, hq * D, k_cache, hkv * D, v_cache, hkv * D, slots3, pool * page)
        up.uniprefill_attention_window_step(p3, q3_out, k_cache, v_cache, hkv * D, kv_len, most * page, table, most, page, window, n_sink, out3, hq * D, lse3, R, ws3, nb3)
        up.uniprefill_linear_attention_step(p3, q3, k3, v3, hkv * D, log_decay, states, hkv * D * D, 2, state_slot, state_slot, y3, hq * D)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    lengths, table_now, left = want["new_len"], want["table"], want["free_left"]
    for _ in range(20):
        for t in (q3, k3, v3):
            t.copy_(_rows(rng, BF, *t.shape)[0])
        before = states.double().cpu().numpy()
        g.replay()
        want = lo.append_pages(lengths, [1, 1], page, table_now, free_host, left, R)
        lengths, table_now, left = want["new_len"], want["table"], want["free_left"]
        np.testing.assert_array_equal(ints(table), table_now)
        np.testing.assert_array_equal(ints(slots3), want["slots"])
        ref, size = lo.norm_rotate(host(q3, hq), w64[0], 1e-6, want["pos"], freq, D, False)
        assert (np.abs(host(q3_out, hq) - ref) <= u * np.abs(ref) + (D + 40) * F * size).all()
        gather = lambda r, n: ao.page_rows(table_now[r].astype(np.int32), n, page)
        o, z, absv, top = lo.window_attention(host(q3_out, hq), host(k_cache, hkv), host(v_cache, hkv), _cu([1, 1]), _cu(lengths), window, n_sink, gather=gather)
        assert (np.abs(host(out3, hq) - o) <= _attention_tolerance(o, absv, top, max(lengths), D, True)).all()
        assert (np.abs(lse3.double().cpu().numpy() - z) <= _lse_tolerance(z, top, max(lengths), D)).all()
        o, pool_now, bound, pbound = lo.linear_attention(host(q3, hq), host(k3, hkv), host(v3, hkv), _cu([1, 1]), ld, before, [1, 0], [1, 0])
        assert (np.abs(host(y3, hq) - o) <= u * np.abs(o) + (D + 515) * F * bound).all()
        assert (np.abs(states.double().cpu().numpy() - pool_now) <= 515 * F * pbound).all()
