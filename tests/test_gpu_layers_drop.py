"""GPU tests of serving behind a drop: pages and positions for a cache that does not hold all tokens of its sequences, and a
prompt whose tokens are dropped, cached in pages and decoded from.

Tolerances as in tests/test_gpu_layers.py; pages and positions are whole numbers and equal."""
import numpy as np
import pytest
import torch

import paper_2605_06221_amd as up
from oracle import attention_oracle as ao
from oracle import layers_oracle as lo
from test_gpu_attention import BF, F, _attention_tolerance, _cu, _dev, _lse_tolerance, _rows, _say
from test_gpu_layers import Pages, _requests

pytestmark = pytest.mark.gpu


class Dropped(Pages):
    """Pages with a number of dropped tokens for every sequence."""

    def __init__(self, *args, dropped=(), **kw):
        self.dropped_host = np.asarray(dropped, np.int32)
        super().__init__(*args, **kw)

    def reset(self):
        super().reset()
        self.dropped = _dev(self.dropped_host)

    def run(self, in_place=False, stream=None):
        return up.uniprefill_append_pages_dropped(
            self.kv_len, self.new, self.dropped, self.n, self.page, self.table, self.table_host.shape[1], self.free, self.num,
            self.num if in_place else self.left, self.kv_len if in_place else self.new_len, self.cu, self.cu_k, self.pos, self.slots, self.capacity,
            self.served, stream=stream)

    def check(self, in_place=False):
        want = lo.append_pages(self.len_host, self.new_host, self.page, self.table_host, self.free_host, self.num_free, self.capacity,
                               self.dropped_host)
        positions = want["pos"]
        got = self.pos.clone()
        plain = lo.append_pages(self.len_host, self.new_host, self.page, self.table_host, self.free_host, self.num_free, self.capacity)
        np.testing.assert_array_equal(got[:self.capacity].cpu().numpy(), np.asarray(positions))
        assert (got[self.capacity:] == -77).all()
        self.pos[:self.capacity] = _dev(np.asarray(plain["pos"], np.int32))      # (the rest as without a drop)
        super().check(in_place)
        self.pos.copy_(got)


@pytest.mark.parametrize("n", [1, 64, 1024, 1025, 4096, 4097])
def test_positions_behind_a_drop(n):
    # one launch (few sequences and tokens), offsets searched in LDS, and in memory
    _say("pages behind a drop", n)
    rng = np.random.default_rng(n)
    dropped = rng.choice([0, 1, 300, 131072, -5, 2 ** 31 - 1], n)
    lengths, new = _requests(n, n, 40)
    for spare in (3, -1):
        b = Dropped(n, lengths, new, 16, spare=spare, dropped=dropped)
        b.run()
        b.check()
    b = Dropped(n, lengths, [1] * n, 16, dropped=dropped, capacity=n + 3)
    b.run(in_place=True)
    b.check(in_place=True)


def test_no_dropped_tokens_is_the_call_without_them():
    _say("pages: the number of dropped tokens left out")
    a = Pages(2, [5, 0, 31], [1, 20, 2], 16)
    b = Dropped(2, [5, 0, 31], [1, 20, 2], 16, dropped=[0, 0, 0])
    b.dropped = None
    a.run()
    b.run()
    for x, y in ((a.table, b.table), (a.pos, b.pos), (a.slots, b.slots), (a.new_len, b.new_len)):
        assert torch.equal(x, y)
    a.check()


def test_a_dropped_prompt_is_cached_and_decoded_from():
    """Two prompts lose tokens in a drop; the layer behind it (norm and rotation into pages, windowed attention over them) runs on what is
    left, then on 40 replayed decode steps.  Every stage against the oracle; what a decode step's query is turned by is the position that
    the token has in its request."""
    _say("a drop, a paged cache behind it, decode steps")
    rng = np.random.default_rng(78)
    hq, hkv, D, page, window, n_sink, hidden_dim = 8, 2, 128, 16, 90, 4, 256
    u = 2.0 ** -8
    lengths = [333, 190]
    R, T = 2, sum(lengths)
    cu_host, ratio = _cu(lengths), np.array([0.3, 0.5], np.float32)
    p = up.make_params(num_seqs=R, total_tokens=T, block_size=32, n_obs=16, n_sink=n_sink, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                       hidden_dim=hidden_dim)

    def host(x, heads):
        return x.double().cpu().numpy().reshape(-1, heads, D)

    # ---- the drop
    q, _ = _rows(rng, BF, T, hq, D)
    k, _ = _rows(rng, BF, T, hkv, D)
    hidden, _ = _rows(rng, BF, T, hidden_dim)
    pos_host = np.concatenate([np.arange(n) for n in lengths]).astype(np.int32)
    _, new_cu_host, kept, nb = up.uniprefill_plan(p, cu_host, ratio)
    hidden_out = torch.zeros(kept, hidden_dim, dtype=BF, device="cuda")
    pos, kept_idx = (torch.zeros(kept, dtype=torch.int32, device="cuda") for _ in range(2))
    new_cu = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    ws = torch.empty(nb + 256, dtype=torch.uint8, device="cuda")
    up.uniprefill_fused(p, q.cuda(), k.cuda(), hidden.cuda(), _dev(pos_host), _dev(cu_host), cu_host, _dev(ratio), ratio, hidden_out, pos, kept_idx,
                        new_cu, None, ws, nb)
    stay = np.diff(new_cu_host)
    assert (stay < lengths).all() and kept == stay.sum()
    np.testing.assert_array_equal(pos.cpu().numpy(), pos_host[kept_idx.cpu().numpy()])
    num_kept = new_cu[1:] - new_cu[:-1]
    num_dropped = _dev(np.asarray(lengths, np.int32)) - num_kept

    # ---- the prompt's retained tokens in the layer behind the drop
    pool, most = 64, 24
    free_host = rng.permutation(pool).astype(np.int32)
    table_host = np.full((R, most), -1, np.int32)
    table, free, num_free = _dev(table_host), _dev(free_host), torch.tensor([pool], dtype=torch.int32, device="cuda")
    kv_len, served, cu, cu_k = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (R, 1, R + 1, R + 1))
    places, slots = torch.zeros(kept, dtype=torch.int32, device="cuda"), torch.zeros(kept, dtype=torch.int64, device="cuda")
    up.uniprefill_append_pages(kv_len, num_kept, R, page, table, most, free, num_free, num_free, kv_len, cu, cu_k, places, slots, kept, served)
    want = lo.append_pages([0, 0], stay, page, table_host, free_host, pool, kept)
    np.testing.assert_array_equal(slots.cpu().numpy(), want["slots"])
    np.testing.assert_array_equal(table.cpu().numpy(), want["table"])
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    freq_dev = _dev(freq)
    w, w64 = _rows(rng, BF, 2, D)
    w = w.cuda()
    k_cache, v_cache = (torch.full((pool * page, hkv * D), float("nan"), dtype=BF, device="cuda") for _ in range(2))

    def check_rotated(got, x64, which, positions):
        ref, size = lo.norm_rotate(x64, w64[which], 1e-6, positions, freq, D, False)
        assert (np.abs(got - ref) <= u * np.abs(ref) + (D + 40) * F * size).all()

    q2, q64 = _rows(rng, BF, kept, hq, D)
    k2, k64 = _rows(rng, BF, kept, hkv, D)
    v2, _ = _rows(rng, BF, kept, hkv, D)
    q2, k2, v2 = (t.cuda() for t in (q2, k2, v2))
    q2_out, out2 = torch.empty_like(q2), torch.empty_like(q2)
    p2 = up.make_params(num_seqs=R, total_tokens=kept, block_size=32, num_q_heads=hq, num_kv_heads=hkv, head_dim=D)
    up.uniprefill_norm_rotate(p2, q2, k2, v2, hkv * D, w[0], w[1], 1e-6, pos, freq_dev, D, 0, None, q2_out, hq * D, k_cache, hkv * D, v_cache, hkv * D,
                              slots, pool * page)
    kept_pos = pos_host[kept_idx.cpu().numpy()]
    check_rotated(host(q2_out, hq), q64, 0, kept_pos)
    check_rotated(host(k_cache, hkv)[want["slots"]], k64, 1, kept_pos)
    _, nb = up.uniprefill_attention_window_plan(p2, new_cu_host, new_cu_host, window, n_sink)
    ws = torch.empty(nb + 256, dtype=torch.uint8, device="cuda")
    up.uniprefill_attention_window(p2, q2_out, k_cache, v_cache, hkv * D, cu, new_cu_host, cu_k, new_cu_host, table, most, page, window, n_sink, out2,
                                   hq * D, None, 0, ws, nb)
    o, _, absv, top = lo.window_attention(host(q2_out, hq), np.nan_to_num(host(k_cache, hkv)), np.nan_to_num(host(v_cache, hkv)), new_cu_host, new_cu_host,
                                          window, n_sink, gather=lambda r, n: ao.page_rows(want["table"][r].astype(np.int32), n, page))
    assert (np.abs(host(out2, hq) - o) <= _attention_tolerance(o, absv, top, int(stay.max()), D, True)).all()

    # ---- decode steps behind the drop, from a graph
    p3 = up.make_params(num_seqs=R, total_tokens=R, block_size=32, num_q_heads=hq, num_kv_heads=hkv, head_dim=D)
    one = torch.ones(R, dtype=torch.int32, device="cuda")
    q3, k3, v3 = (torch.zeros(R, h * D, dtype=BF, device="cuda") for h in (hq, hkv, hkv))
    q3_out, out3, lse3 = torch.zeros_like(q3), torch.zeros_like(q3), torch.zeros(hq, R, device="cuda")
    _, nb3 = up.uniprefill_attention_window_step_plan(p3, most * page, window, n_sink)
    ws3 = torch.empty(nb3 + 256, dtype=torch.uint8, device="cuda")
    pos3, slots3 = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, dtype=torch.int64, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        up.uniprefill_append_pages_dropped(kv_len, one, num_dropped, R, page, table, most, free, num_free, num_free, kv_len, cu, cu_k, pos3, slots3, R,
                                           served)
        up.uniprefill_norm_rotate(p3, q3, k3, v3, hkv * D, w[0], w[1], 1e-6, pos3, freq_dev, D, 0, None, q3_out, hq * D, k_cache, hkv * D, v_cache,
                                  hkv * D, slots3, pool * page)
        up.uniprefill_attention_window_step(p3, q3_out, k_cache, v_cache, hkv * D, kv_len, most * page, table, most, page, window, n_sink, out3,
                                            hq * D, lse3, R, ws3, nb3)
    for i in range(40):
        for t in (q3, k3, v3):
            t.copy_(_rows(rng, BF, *t.shape)[0])
        g.replay()
        want = lo.append_pages(want["new_len"], [1, 1], page, want["table"], free_host, want["free_left"], R)
        np.testing.assert_array_equal(table.cpu().numpy(), want["table"])
        np.testing.assert_array_equal(slots3.cpu().numpy(), want["slots"])
        positions = [n + i for n in lengths]      # the request's next position, whatever its cache holds
        np.testing.assert_array_equal(pos3.cpu().numpy(), positions)
        check_rotated(host(q3_out, hq), host(q3, hq), 0, positions)
        check_rotated(host(k_cache, hkv)[want["slots"]], host(k3, hkv), 1, positions)
        o, z, absv, top = lo.window_attention(host(q3_out, hq), np.nan_to_num(host(k_cache, hkv)), np.nan_to_num(host(v_cache, hkv)), _cu([1, 1]),
                                              _cu(want["new_len"]), window, n_sink,
                                              gather=lambda r, n: ao.page_rows(want["table"][r].astype(np.int32), n, page))
        longest = max(want["new_len"])
        assert (np.abs(host(out3, hq) - o) <= _attention_tolerance(o, absv, top, longest, D, True)).all()
        assert (np.abs(lse3.double().cpu().numpy() - z) <= _lse_tolerance(z, top, longest, D)).all()
