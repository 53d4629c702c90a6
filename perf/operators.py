"""Timing cases of the attention layer's operators and of the 4-bit KV cache, through the public entry points.

  attention  uniprefill_attention            causal attention of a packed batch with its log-sum-exp, what the scoring of
                                             a drop layer is fed with; own keys, or earlier context in a paged cache
  store      uniprefill_cache_store_q4       key and value rows into slots of a 4-bit cache, and back out of it
             uniprefill_cache_load_q4        (what the next chunk's attention and scoring read)
  decode     uniprefill_attention_q4         one query token per sequence over the 4-bit cache, optionally with the
                                             attention weight that every cached token has accumulated
  evict      uniprefill_cache_evict          shrink the sequences' caches to a budget by that accumulated weight

Shapes are those of the repository's workloads and tests: 8/8, 32/8, 40/8 and 16/4 heads, head dimension 64, 128 and
256, 16-token pages, prompts of one to some ten thousand tokens, caches to 131072.  Rows are normal in bf16 (a few cases
float32); keys are scaled by exp(spread * z), z ~ N(0,1), as attention over text is concentrated on few tokens.
"""
import math

import numpy as np
import torch

own = False

GROUP = 64             # elements that share one (lowest value, step) pair in the 4-bit cache
N_SINK = 128
N_RECENT = 128

_DEFAULTS = {"op": "attention", "lengths": "1000", "earlier": "", "q_heads": 32, "kv_heads": 8, "head_dim": 128,
             "dtype": "bf16", "page": 16, "spread": 0.5, "mass": False, "budget": 0, "cache": "bf16"}


def _case(name, **kw):
    return {"name": name, **_DEFAULTS, **kw}


def listed():
    return [
        # the smallest prompt worth sparsifying, float32 operands: launches and host time, hardly any work
        _case("attn_short_f32", lengths="1000", q_heads=8, dtype="f32", spread=0.0),
        # one 32768-token prompt of an 8B-shaped layer
        _case("attn_prompt_32k", lengths="32768"),
        # narrow heads, a ragged batch of prompts from one token on
        _case("attn_ragged_head_64", lengths="12289,1,24576,7011,300,63,2050", head_dim=64, spread=1.0),
        # wide heads, one prompt
        _case("attn_head_256", lengths="16384", head_dim=256, q_heads=16, spread=1.0),
        # continuous batch: 48 decode rows and two prefill chunks, everything earlier in a paged cache
        _case("attn_mixed_paged", lengths="48*1,8192,3001", earlier="24*6001,24*1500,57344,5000"),
        # one decode step of 64 sequences enters the cache
        _case("store_64", op="store", lengths="64*1"),
        # a 131072-token prompt enters the cache and is read back
        _case("store_128k", op="store", lengths="131072"),
        # one sequence, a short cache: latency
        _case("decode_1000", op="decode", lengths="1000", spread=0.0),
        # a decode step of 48 sequences, weights accumulated for a later eviction; one slot of the batch is unused
        _case("decode_48_mass", op="decode", mass=True,
              lengths="0,16211,15,9999,28174,21619,17691,10340,11489,3342,4362,2547,7443,27028,21841,30103,24*6001,8*1500"),
        # one sequence with a long context, weights accumulated as well
        _case("decode_128k", op="decode", lengths="131072", q_heads=40, spread=1.0, mass=True),
        # a short cache in bf16 shrinks to a quarter
        _case("evict_4096", op="evict", lengths="4096", budget=1024),
        # sixteen caches of ragged lengths in 4 bits shrink to at most 8192 tokens
        _case("evict_16_ragged", op="evict", cache="q4", budget=8192,
              lengths="28174,21619,17691,10340,11489,3342,4362,2547,7443,27028,21841,30103,17444,20703,32420,18019"),
    ]


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        top = most.setdefault((c["op"], c["dtype"]), {"bytes": 0, "flops": 0})
        top["bytes"], top["flops"] = max(top["bytes"], w["bytes"]), max(top["flops"], w["flops"])
    most["attention", "f32"] = {"bytes": 4 << 30, "flops": 3e11}
    for _ in range(1000):
        op = rng.choice(["attention", "attention", "store", "decode", "decode", "evict"])
        top_len = {"attention": 40000, "store": 131072, "decode": 131072, "evict": 200000}[op]
        total = int(round(math.exp(rng.uniform(math.log(20), math.log(top_len)))))
        n_seqs = 1 if rng.random() < 0.4 else rng.randint(2, 24)
        cuts = sorted(rng.randint(1, max(1, total - 1)) for _ in range(n_seqs - 1))
        lengths = [b - a for a, b in zip([0] + cuts, cuts + [total]) if b > a]
        q_heads, kv_heads = rng.choice([(8, 8), (32, 8), (32, 8), (40, 8), (16, 4)])
        c = {**_DEFAULTS, "op": op, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": rng.choice([64, 128, 128, 128, 256]),
             "page": rng.choice([16, 16, 32, 64, 128]), "spread": rng.choice([0.0, 0.5, 1.0])}
        if op == "attention":
            if rng.random() < 0.15:
                c["dtype"] = "f32"
                c["head_dim"] = rng.choice([64, 128])
            if rng.random() < 0.25:
                lengths = [1] * rng.randint(1, 64) + lengths
            if rng.random() < 0.4:
                c["earlier"] = ",".join(str(int(math.exp(rng.uniform(math.log(20), math.log(40000))))) for _ in lengths)
        elif op == "decode":
            lengths = [max(0, n + rng.randint(-1, 1)) for n in lengths]
            c["mass"] = rng.random() < 0.5
        elif op == "evict":
            c["cache"] = rng.choice(["bf16", "q4"])
            c["budget"] = max(N_SINK + N_RECENT, int(max(lengths) * rng.uniform(0.1, 1.1)))
        c["lengths"] = ",".join(str(n) for n in lengths)
        w, top = work(c), most.get((op, c["dtype"]))
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] and sum(_keys(c)) <= 300000:
            return c
    raise RuntimeError("no case of the range fits")


def _numbers(text):
    out = []
    for part in filter(None, text.split(",")):
        count, _, value = part.rpartition("*")
        out += [int(value)] * (int(count) if count else 1)
    return out


def _keys(case):
    """Keys of every sequence: its own tokens' and those before them."""
    lengths = _numbers(case["lengths"])
    earlier = _numbers(case["earlier"]) or [0] * len(lengths)
    return [n + e for n, e in zip(lengths, earlier)]


def _row_bytes(case):
    """Bytes of one token in a cache of keys (or of values): all kv heads."""
    if case["op"] == "decode" or case["op"] == "store" or case["cache"] == "q4":
        return case["kv_heads"] * (case["head_dim"] // 2 + 4 * case["head_dim"] // GROUP)
    return case["kv_heads"] * case["head_dim"] * 2


def work(case):
    lengths, keys, d = _numbers(case["lengths"]), _keys(case), case["head_dim"]
    hq, hkv, e = case["q_heads"], case["kv_heads"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "attention":
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(lengths, keys))
        return {"bytes": sum(lengths) * hq * (2 * d * e + 4) + 2 * sum(keys) * hkv * d * e, "flops": 4 * d * hq * pairs}
    if case["op"] == "store":
        # rows in, cache out, cache in, rows out; keys and values
        return {"bytes": sum(lengths) * (2 * (2 * hkv * d * e + 2 * _row_bytes(case)) + 8), "flops": 0}
    if case["op"] == "decode":
        return {"bytes": sum(lengths) * (2 * _row_bytes(case) + (8 if case["mass"] else 0)) + len(lengths) * hq * (4 * d + 4),
                "flops": 4 * d * hq * sum(lengths)}
    kept = sum(min(n, case["budget"]) for n in lengths)
    reread = 2 * kept * (_row_bytes(case) + 2 * hkv * d) if case["cache"] == "q4" else 0
    return {"bytes": kept * (4 * _row_bytes(case) + 8) + 4 * sum(lengths) + reread, "flops": 0}


# ---------------------------------------------------------------------------------------------------- inputs
def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _normal(gen, dtype, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _key_rows(gen, dtype, n, heads, d, spread):
    k = _normal(gen, dtype, n, heads, d)
    if spread:
        z = torch.randn(n, generator=gen, device="cuda")
        for lo in range(0, n, 1 << 15):
            part = k[lo:lo + (1 << 15)]
            part.copy_(part.float() * torch.exp(spread * z[lo:lo + (1 << 15), None, None]))
    return k


def _block_table(gen, lengths, page, first=0):
    """Pages of every sequence in random order of the pool [first, first + pages), and the pool's page count."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(need), generator=gen, device="cuda") + first
    table = torch.zeros(len(lengths), max(need + [1]), dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n].to(torch.int32)
        at += n
    return table, sum(need)


def _slots(table, r, n, page):
    i = torch.arange(n, device="cuda")
    return table[r].long()[i // page] * page + i % page


def _quantise(x):
    """Codes 0..15 and (lowest value, step) of every 64 elements of x [n, heads, d]; 64 bits where a border decides."""
    g = x.double().reshape(x.shape[0], x.shape[1], -1, GROUP)
    lo = _bf16_below(g.amin(-1).float())
    step = _bf16_above((g.amax(-1) - lo.double()) / 15)
    code = torch.round((g - lo.double()[..., None]) / step.double()[..., None]).nan_to_num(0.0).clamp(0, 15)
    return code.to(torch.uint8).reshape(x.shape), lo, step


def _bf16_below(x):
    """Largest bf16 not above x (float32)."""
    b = x.contiguous().view(torch.int32).long() & 0xFFFFFFFF
    b = torch.where(b >= 1 << 31, b + 0xFFFF, b) & 0xFFFF0000
    return (b - ((b >> 31) << 32)).to(torch.int32).view(torch.float32).to(torch.bfloat16)


def _bf16_above(x):
    """Smallest bf16 not below x >= 0 (float64)."""
    b = x.float().contiguous().view(torch.int32) & -65536
    y = b.view(torch.float32)
    return torch.where(y.double() < x, (b + 65536).view(torch.float32), y).to(torch.bfloat16)


def _pack(code, lo, step, row_stride):
    """Rows of the 4-bit cache: every head's codes, low nibble first, then every head's (lowest value, step) pairs."""
    n = code.shape[0]
    nib = code.reshape(n, -1, 2)
    pairs = torch.stack([lo.reshape(n, -1), step.reshape(n, -1)], dim=2).contiguous().view(torch.uint8).reshape(n, -1)
    rows = torch.zeros(n, row_stride, dtype=torch.uint8, device="cuda")
    body = torch.cat([nib[:, :, 0] | (nib[:, :, 1] << 4), pairs], dim=1)
    rows[:, :body.shape[1]] = body
    return rows


def _unpack(rows, heads, d):
    """float32 values [n, heads, d] of rows of the 4-bit cache."""
    n, half = rows.shape[0], heads * d // 2
    code = torch.stack([rows[:, :half] & 15, rows[:, :half] >> 4], dim=2).reshape(n, heads, d // GROUP, GROUP).float()
    pair = rows[:, half:half + heads * d // GROUP * 4].contiguous().view(torch.bfloat16).float().reshape(n, heads, d // GROUP, 2)
    return (pair[..., :1] + pair[..., 1:] * code).reshape(n, heads, d)


def _row_stride(case):
    return -(-_row_bytes(case) // 16) * 16


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lengths, keys = _numbers(case["lengths"]), _keys(case)
    s = {**{k: case[k] for k in ("op", "q_heads", "kv_heads", "head_dim", "page", "mass", "budget", "cache")},
         "lengths": lengths, "keys": keys, "scale": 1.0 / math.sqrt(case["head_dim"]),
         "dtype": torch.float32 if case["dtype"] == "f32" else torch.bfloat16}
    {"attention": _prepare_attention, "store": _prepare_store, "decode": _prepare_decode, "evict": _prepare_evict}[case["op"]](
        s, case, gen)
    return s


def _params(s, seqs, tokens):
    import paper_2605_06221_amd as up
    return up.make_params(num_seqs=seqs, total_tokens=tokens, block_size=64, num_q_heads=s["q_heads"], num_kv_heads=s["kv_heads"],
                          head_dim=s["head_dim"], qk_dtype=up.UP_F32 if s["dtype"] == torch.float32 else up.UP_BF16)


def _prepare_attention(s, case, gen):
    lengths, keys, page, dt = s["lengths"], s["keys"], s["page"], s["dtype"]
    hkv, d, tokens = s["kv_heads"], s["head_dim"], sum(s["lengths"])
    s["q"] = _normal(gen, dt, tokens, s["q_heads"], d)
    k = _key_rows(gen, dt, sum(keys), hkv, d, case["spread"])
    v = _normal(gen, dt, sum(keys), hkv, d)
    s["cu_host"], s["cu_k_host"] = _offsets(lengths), _offsets(keys)
    s["cu"], s["cu_k"] = torch.from_numpy(s["cu_host"]).cuda(), torch.from_numpy(s["cu_k_host"]).cuda()
    s["table"] = None
    if case["earlier"]:
        s["table"], pages = _block_table(gen, keys, page)
        kc = torch.zeros(pages * page, hkv, d, dtype=dt, device="cuda")
        vc = torch.zeros_like(kc)
        for r, n in enumerate(keys):
            at = _slots(s["table"], r, n, page)
            kc[at], vc[at] = k[s["cu_k_host"][r]:s["cu_k_host"][r + 1]], v[s["cu_k_host"][r]:s["cu_k_host"][r + 1]]
        k, v = kc, vc
    s["k"], s["v"] = k, v
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q_heads"], tokens, device="cuda")
    if own:
        import paper_2605_06221_amd as up
        s["p"] = _params(s, len(lengths), tokens)
        _, s["ws_bytes"] = up.uniprefill_attention_plan(s["p"], s["cu_host"], s["cu_k_host"] if s["table"] is not None else None)
        s["ws"] = torch.empty(s["ws_bytes"] + 256, dtype=torch.uint8, device="cuda")


def _prepare_store(s, case, gen):
    n, hkv, d = sum(s["lengths"]), s["kv_heads"], s["head_dim"]
    s["k"] = _key_rows(gen, s["dtype"], n, hkv, d, case["spread"])
    s["v"] = _normal(gen, s["dtype"], n, hkv, d)
    # every sequence's tokens follow 5 cached ones: its first slot lies inside a page
    table, pages = _block_table(gen, [m + 5 for m in s["lengths"]], s["page"])
    s["slots"] = torch.cat([_slots(table, r, m + 5, s["page"])[5:] for r, m in enumerate(s["lengths"])])
    s["stride"], s["num_slots"] = _row_stride(case), pages * s["page"]
    s["k_cache"] = torch.zeros(s["num_slots"], s["stride"], dtype=torch.uint8, device="cuda")
    s["v_cache"] = torch.zeros_like(s["k_cache"])
    s["k_out"], s["v_out"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    if own:
        s["p"] = _params(s, 1, n)


def _fill_q4(s, case, gen):
    """A pool of pages that holds the sequences' keys and values in 4 bits."""
    s["table"], s["pages"] = _block_table(gen, s["lengths"], s["page"])
    s["stride"] = _row_stride(case)
    extra = sum(-(-min(n, s["budget"]) // s["page"]) for n in s["lengths"])
    s["k_cache"] = torch.zeros((s["pages"] + extra) * s["page"], s["stride"], dtype=torch.uint8, device="cuda")
    s["v_cache"] = torch.zeros_like(s["k_cache"])
    for r, n in enumerate(s["lengths"]):
        at = _slots(s["table"], r, n, s["page"])
        for cache, spread in ((s["k_cache"], case["spread"]), (s["v_cache"], 0.0)):
            for lo in range(0, n, 1 << 14):
                rows = _key_rows(gen, torch.bfloat16, min(n - lo, 1 << 14), s["kv_heads"], s["head_dim"], spread)
                cache[at[lo:lo + rows.shape[0]]] = _pack(*_quantise(rows), s["stride"])


def _masses(gen, s):
    """Weight accumulated per cached token: most of it on few tokens, none on many."""
    most = max(s["lengths"] + [1])
    z = torch.randn(len(s["lengths"]), most, generator=gen, device="cuda")
    return torch.where(torch.rand(z.shape, generator=gen, device="cuda") < 0.3, torch.zeros_like(z), torch.exp(2.5 * z - 8))


def _prepare_decode(s, case, gen):
    n_seqs = len(s["lengths"])
    _fill_q4(s, case, gen)
    s["q"] = _normal(gen, torch.bfloat16, n_seqs, s["q_heads"], s["head_dim"])
    s["kv_len"] = torch.tensor(s["lengths"], dtype=torch.int32, device="cuda")
    s["mass_in"] = _masses(gen, s) if case["mass"] else None
    s["mass_out"] = torch.zeros_like(s["mass_in"]) if case["mass"] else None
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q_heads"], n_seqs, device="cuda")
    if own:
        import paper_2605_06221_amd as up
        s["p"] = _params(s, n_seqs, n_seqs)
        s["max_len"] = max(s["lengths"])
        _, s["ws_bytes"] = up.uniprefill_attention_q4_plan(s["p"], s["max_len"], case["mass"])
        s["ws"] = torch.empty(s["ws_bytes"] + 256, dtype=torch.uint8, device="cuda")


def _prepare_evict(s, case, gen):
    kept = [min(n, s["budget"]) for n in s["lengths"]]
    if case["cache"] == "q4":
        _fill_q4(s, case, gen)
    else:
        s["table"], s["pages"] = _block_table(gen, s["lengths"], s["page"])
        extra = sum(-(-n // s["page"]) for n in kept)
        s["k_cache"] = _normal(gen, torch.bfloat16, (s["pages"] + extra) * s["page"], s["kv_heads"], s["head_dim"])
        s["v_cache"] = _normal(gen, torch.bfloat16, (s["pages"] + extra) * s["page"], s["kv_heads"], s["head_dim"])
        s["k_cache"][s["pages"] * s["page"]:].zero_()
        s["v_cache"][s["pages"] * s["page"]:].zero_()
    # pages for what stays, from another part of the pool
    s["new_table"], _ = _block_table(gen, kept, s["page"], first=s["pages"])
    s["new_slots"] = torch.cat([_slots(s["new_table"], r, n, s["page"]) for r, n in enumerate(kept)])
    n_seqs = len(s["lengths"])
    s["kv_len"] = torch.tensor(s["lengths"], dtype=torch.int32, device="cuda")
    s["mass"] = _masses(gen, s)
    s["mass_out"] = torch.zeros(n_seqs, s["budget"], device="cuda")
    s["kept_idx"] = torch.zeros(n_seqs, s["budget"], dtype=torch.int32, device="cuda")
    s["new_len"] = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
    s["max_len"] = max(s["lengths"])
    if case["cache"] == "q4":
        s["k_out"] = torch.zeros(sum(kept), s["kv_heads"], s["head_dim"], dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
    if own:
        s["p"] = _params(s, n_seqs, sum(kept))


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return {"attention": _own_attention, "store": _own_store, "decode": _own_decode, "evict": _own_evict}[s["op"]](s)
    return {"attention": _plain_attention, "store": _plain_store, "decode": _plain_decode, "evict": _plain_evict}[s["op"]](s)


def _own_attention(s):
    import paper_2605_06221_amd as up
    hq, hkv, d, paged = s["q_heads"], s["kv_heads"], s["head_dim"], s["table"] is not None
    up.uniprefill_attention(s["p"], s["q"], s["k"], s["v"], hkv * d, s["cu"], s["cu_host"], s["cu_k"] if paged else None,
                            s["cu_k_host"] if paged else None, s["table"], s["table"].shape[1] if paged else 0, s["page"],
                            s["out"], hq * d, s["lse"], s["lse"].shape[1], s["ws"], s["ws_bytes"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_store(s):
    import paper_2605_06221_amd as up
    n, row = s["slots"].shape[0], s["kv_heads"] * s["head_dim"]
    up.uniprefill_cache_store_q4(s["p"], s["k"], s["v"], row, s["slots"], n, None, s["k_cache"], s["v_cache"], s["stride"],
                                 s["num_slots"])
    up.uniprefill_cache_load_q4(s["p"], s["k_cache"], s["v_cache"], s["stride"], s["num_slots"], s["slots"], n, None, s["k_out"],
                                s["v_out"], row)
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_decode(s):
    import paper_2605_06221_amd as up
    mass = s["mass_out"] is not None
    up.uniprefill_attention_q4(s["p"], s["q"], s["k_cache"], s["v_cache"], s["stride"], s["kv_len"], s["max_len"], s["table"],
                               s["table"].shape[1], s["page"], s["out"], s["q_heads"] * s["head_dim"], s["lse"],
                               s["lse"].shape[1], s["mass_in"], s["mass_out"], s["mass_out"].shape[1] if mass else 0, s["ws"],
                               s["ws_bytes"])
    return {"out": s["out"], "lse": s["lse"], **({"mass": s["mass_out"]} if mass else {})}


def _own_evict(s):
    import paper_2605_06221_amd as up
    row = s["stride"] if s["cache"] == "q4" else s["kv_heads"] * s["head_dim"] * 2
    up.uniprefill_cache_evict(s["k_cache"], s["v_cache"], row, row, s["mass"], s["mass"].shape[1], s["kv_len"], len(s["lengths"]),
                              s["max_len"], s["budget"], N_SINK, N_RECENT, s["table"], s["table"].shape[1], s["new_table"],
                              s["new_table"].shape[1], s["page"], s["kept_idx"], s["mass_out"], s["budget"], s["new_len"])
    if s["cache"] == "q4":
        # what the next chunk of the sequences attends to
        up.uniprefill_cache_load_q4(s["p"], s["k_cache"], s["v_cache"], s["stride"], s["k_cache"].shape[0], s["new_slots"],
                                    s["new_slots"].shape[0], None, s["k_out"], s["v_out"], s["kv_heads"] * s["head_dim"])
    return _evicted(s)


def _evicted(s):
    if s["cache"] == "q4":
        rows = {"k": s["k_out"], "v": s["v_out"]}
    else:
        rows = {"k": s["k_cache"][s["pages"] * s["page"]:], "v": s["v_cache"][s["pages"] * s["page"]:]}
    return {**rows, "kept_idx": s["kept_idx"], "mass": s["mass_out"], "new_len": s["new_len"]}


def _plain_attention(s):
    group = s["q_heads"] // s["kv_heads"]
    for r, (n, keys) in enumerate(zip(s["lengths"], s["keys"])):
        if s["table"] is not None:
            at = _slots(s["table"], r, keys, s["page"])
        else:
            at = slice(int(s["cu_k_host"][r]), int(s["cu_k_host"][r + 1]))
        q0, first = int(s["cu_host"][r]), keys - n
        chunk = max(1, (1 << 28) // (keys * group))
        for h in range(s["kv_heads"]):
            k, v = s["k"][at, h].float(), s["v"][at, h].float()
            heads = slice(h * group, (h + 1) * group)
            for lo in range(0, n, chunk):
                hi = min(n, lo + chunk)
                seen = first + hi
                q = s["q"][q0 + lo:q0 + hi, heads].float().reshape(-1, s["head_dim"])
                x = (q @ k[:seen].t().contiguous()).reshape(hi - lo, group, seen) * s["scale"]
                later = torch.arange(seen, device="cuda")[None, :] > torch.arange(first + lo, first + hi, device="cuda")[:, None]
                x.masked_fill_(later[:, None, :], -math.inf)
                top = x.amax(2, keepdim=True)
                x = x.sub_(top).exp_()
                total = x.sum(2, keepdim=True)
                o = (x.reshape(-1, seen) @ v[:seen]).reshape(hi - lo, group, -1) / total
                s["out"][q0 + lo:q0 + hi, heads] = o.to(s["out"].dtype)
                s["lse"][heads, q0 + lo:q0 + hi] = (top + torch.log(total))[:, :, 0].t()
    return {"out": s["out"], "lse": s["lse"]}


def _plain_store(s):
    for x, cache, out in ((s["k"], s["k_cache"], s["k_out"]), (s["v"], s["v_cache"], s["v_out"])):
        for lo in range(0, x.shape[0], 1 << 15):
            at = s["slots"][lo:lo + (1 << 15)]
            cache[at] = _pack(*_quantise(x[lo:lo + (1 << 15)]), s["stride"])
            out[lo:lo + (1 << 15)] = _unpack(cache[at], s["kv_heads"], s["head_dim"]).to(out.dtype)
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_decode(s):
    hkv, d, group = s["kv_heads"], s["head_dim"], s["q_heads"] // s["kv_heads"]
    if s["mass_out"] is not None:
        s["mass_out"].zero_()
    for r, n in enumerate(s["lengths"]):
        if n == 0:
            s["out"][r] = 0
            s["lse"][:, r] = -math.inf
            continue
        at = _slots(s["table"], r, n, s["page"])
        k = _unpack(s["k_cache"][at], hkv, d).permute(1, 2, 0).contiguous()
        v = _unpack(s["v_cache"][at], hkv, d).permute(1, 0, 2).contiguous()
        x = torch.matmul(s["q"][r].float().reshape(hkv, group, d), k) * s["scale"]
        top = x.amax(2, keepdim=True)
        w = torch.exp(x - top)
        total = w.sum(2, keepdim=True)
        s["out"][r] = (torch.matmul(w, v) / total).reshape(-1, d).to(s["out"].dtype)
        s["lse"][:, r] = (top + torch.log(total)).reshape(-1)
        if s["mass_out"] is not None:
            s["mass_out"][r, :n] = s["mass_in"][r, :n] + (w / total).reshape(-1, n).sum(0) / s["q_heads"]
    return {"out": s["out"], "lse": s["lse"], **({"mass": s["mass_out"]} if s["mass_out"] is not None else {})}


def _kept_tokens(mass, n, budget):
    """Indices that stay, ascending: sinks, recent tokens, then the largest masses (equal ones: the lower index)."""
    if n <= budget:
        return torch.arange(n, device="cuda")
    key = mass[:n].clone()
    key[:N_SINK] = math.inf
    key[n - N_RECENT:] = math.inf
    return torch.sort(key, descending=True, stable=True).indices[:budget].sort().values


def _plain_evict(s):
    at_out = 0
    for r, n in enumerate(s["lengths"]):
        kept = _kept_tokens(s["mass"][r], n, s["budget"])
        m = kept.shape[0]
        src, dst = _slots(s["table"], r, n, s["page"])[kept], _slots(s["new_table"], r, m, s["page"])
        for cache in (s["k_cache"], s["v_cache"]):
            cache[dst] = cache[src]
        s["kept_idx"][r, :m], s["mass_out"][r, :m], s["new_len"][r] = kept.to(torch.int32), s["mass"][r][kept], m
        if s["cache"] == "q4":
            s["k_out"][at_out:at_out + m] = _unpack(s["k_cache"][dst], s["kv_heads"], s["head_dim"]).to(torch.bfloat16)
            s["v_out"][at_out:at_out + m] = _unpack(s["v_cache"][dst], s["kv_heads"], s["head_dim"]).to(torch.bfloat16)
        at_out += m
    return _evicted(s)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "store": _exact_store, "decode": _exact_decode, "evict": _exact_evict}[s["op"]](s)


def _softmax_sum(q, k, v, scale, visible):
    """Rows q [n, d] over keys [m, d]: attention output and log-sum-exp, the keys a row does not see masked out."""
    x = torch.mm(q, k.T.contiguous()) * scale
    if visible is not None:
        x = torch.where(visible, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, dim=1)
    x = torch.exp(x - lse[:, None])
    return torch.mm(x, v), lse, x


def _exact_attention(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for r in range(len(s["lengths"])):
        n, m = s["lengths"][r], s["keys"][r]
        base = sum(s["lengths"][:r])
        if s["table"] is None:
            rows = torch.arange(m, device="cuda") + sum(s["keys"][:r])
        else:
            rows = (s["table"][r].long()[:, None] * s["page"] + torch.arange(s["page"], device="cuda")).reshape(-1)[:m]
        for hq in range(s["q_heads"]):
            hk = hq * s["kv_heads"] // s["q_heads"]
            k, v = s["k"][rows, hk].double(), s["v"][rows, hk].double()
            for a in range(0, n, 4096):
                b = min(n, a + 4096)
                pos = torch.arange(m - n + a, m - n + b, device="cuda")
                visible = torch.arange(m, device="cuda")[None] <= pos[:, None]
                o, z, _ = _softmax_sum(s["q"][base + a:base + b, hq].double(), k, v, s["scale"], visible)
                out[base + a:base + b, hq], lse[hq, base + a:base + b] = o, z
    return {"out": out, "lse": lse}


def _values64(x):
    """What the 4-bit cache stands for, from the rows that went into it."""
    out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
    for g in range(0, x.shape[2], GROUP):
        part = x[:, :, g:g + GROUP].double()
        low = part.min(dim=2, keepdim=True).values
        low16 = low.bfloat16().double()
        low16 = torch.where(low16 > low, _next16(low16, -1), low16)
        want = (part.max(dim=2, keepdim=True).values - low16) / 15
        step = want.bfloat16().double()
        step = torch.where(step < want, _next16(step, 1), step)
        code = torch.where(step > 0, torch.round((part - low16) / step), torch.zeros_like(part))
        out[:, :, g:g + GROUP] = low16 + step * code.clamp(max=15)
    return out


def _next16(x, way):
    """The bf16 value next to x (a bf16 value held in 64 bits): above (1) or below (-1)."""
    bits = x.bfloat16().view(torch.int16)
    up = (x >= 0) if way > 0 else (x > 0)
    return torch.where(up, bits + way, bits - way).view(torch.bfloat16).double()


def _exact_store(s):
    return {"k": _values64(s["k"]), "v": _values64(s["v"])}


def _read64(cache, rows, heads, d):
    """Values of cache rows: byte j of a head holds elements 2j (low half) and 2j + 1; the pairs follow all heads' codes."""
    raw = cache[rows].cpu().numpy()
    codes = np.empty((raw.shape[0], heads * d))
    codes[:, 0::2], codes[:, 1::2] = raw[:, :heads * d // 2] % 16, raw[:, :heads * d // 2] // 16
    words = raw[:, heads * d // 2:heads * d // 2 + heads * d // 16].copy().view(np.uint16).astype(np.uint32) << 16
    pair = words.view(np.float32).astype(np.float64).reshape(raw.shape[0], -1, 2)
    return torch.from_numpy((pair[:, :, :1] + pair[:, :, 1:] * codes.reshape(raw.shape[0], -1, GROUP)).reshape(-1, heads, d)).cuda()


def _exact_decode(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    mass = None if s["mass_in"] is None else torch.zeros(s["mass_in"].shape, dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["lengths"]):
        if n == 0:
            continue
        rows = (s["table"][r].long()[:, None] * s["page"] + torch.arange(s["page"], device="cuda")).reshape(-1)[:n]
        k = _read64(s["k_cache"], rows, s["kv_heads"], s["head_dim"])
        v = _read64(s["v_cache"], rows, s["kv_heads"], s["head_dim"])
        weight = torch.zeros(n, dtype=torch.float64, device="cuda")
        for hq in range(s["q_heads"]):
            hk = hq * s["kv_heads"] // s["q_heads"]
            o, z, w = _softmax_sum(s["q"][r, hq][None].double(), k[:, hk], v[:, hk].contiguous(), s["scale"], None)
            out[r, hq], lse[hq, r] = o[0], z[0]
            weight += w[0]
        if mass is not None:
            mass[r, :n] = s["mass_in"][r, :n].double() + weight / s["q_heads"]
    return {"out": out, "lse": lse, **({"mass": mass} if mass is not None else {})}


def _exact_evict(s):
    idx, mass, new_len = torch.zeros_like(s["kept_idx"]).cpu(), torch.zeros(s["mass_out"].shape, dtype=torch.float64), []
    weights = s["mass"].cpu().numpy()
    src, dst = [], []
    for r, n in enumerate(s["lengths"]):
        forced = set(range(min(n, N_SINK))) | set(range(max(0, n - N_RECENT), n))
        rest = np.array([i for i in range(n) if i not in forced], dtype=np.int64)
        room = max(0, min(n, s["budget"]) - len(forced))
        best = rest[np.lexsort((rest, -weights[r][rest]))][:room]
        kept = np.array(sorted(forced | set(best.tolist())), dtype=np.int64)
        idx[r, :len(kept)] = torch.from_numpy(kept.astype(np.int32))
        mass[r, :len(kept)] = torch.from_numpy(weights[r][kept].astype(np.float64))
        new_len.append(len(kept))
        old, new = s["table"][r].cpu().numpy().astype(np.int64), s["new_table"][r].cpu().numpy().astype(np.int64)
        j = np.arange(len(kept))
        src.append(old[kept // s["page"]] * s["page"] + kept % s["page"])
        dst.append(new[j // s["page"]] * s["page"] + j % s["page"])
    src, dst = torch.from_numpy(np.concatenate(src)).cuda(), torch.from_numpy(np.concatenate(dst)).cuda()
    rows = {}
    for name in ("k", "v"):
        cache = s[name + "_cache"]
        if s["cache"] == "q4":
            rows[name] = _read64(cache, src, s["kv_heads"], s["head_dim"])
        else:
            moved = torch.zeros(cache[s["pages"] * s["page"]:].shape, dtype=torch.float64, device="cuda")
            moved[dst - s["pages"] * s["page"]] = cache[src].double()
            rows[name] = moved
    return {**rows, "kept_idx": idx.cuda(), "mass": mass.cuda(), "new_len": torch.tensor(new_len, dtype=torch.int32, device="cuda")}
