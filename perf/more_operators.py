"""Timing cases of the operators that the layers between two drops are made of, through the public entry points.

  window   uniprefill_attention_window       causal attention in which a token sees the last `window` tokens and the first
                                             `n_sink` ones: prompts, ragged batches, chunks over a paged cache
  step     uniprefill_attention_window_step  the same for one new token per sequence over a paged cache, lengths on the device
  linear   uniprefill_linear_attention       attention without a softmax, with a decay for each kv head and a state that the
                                             sequence carries: prompts and chunks, whatever state they continue from
  state    uniprefill_linear_attention_step  the same for one new token per sequence
  rotate   uniprefill_norm_rotate            norm of every query and key head and rotation by its position in one pass, keys and
                                             values straight into the slots of a paged cache
  pages    uniprefill_append_pages           pages for a step's new tokens: block table, slots, positions and offsets from the
                                             requests' lengths

Shapes are those of the repository's workloads and tests: 8/8, 32/8, 40/8 and 16/4 heads (32/32 as well where there is a state),
head dimension 64, 128 and 256, 16-token pages, prompts of one to some ten thousand tokens, caches to 131072.
"""
import math

import numpy as np
import torch

own = False

_DEFAULTS = {"op": "window", "lengths": "1000", "earlier": "", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "dtype": "bf16",
             "page": 16, "window": 1024, "n_sink": 4, "decay": 1.0, "rot_dim": 128, "norm": True, "pairs": False, "spare": 4}


def _case(name, **kw):
    return {"name": name, **_DEFAULTS, **kw}


def listed():
    return [
        # one prompt of an 8B-shaped layer, a window of an eighth of it, the drop's sinks kept visible
        _case("window_prompt_32k", lengths="32768", window=4096, n_sink=128),
        # narrow heads, a ragged batch of chunks, most of them behind cached context, a window that no tile divides
        _case("window_ragged_head_64", lengths="12289,1,9000,7011,300,63,2050", earlier="0,20001,5,777,40000,999,1000",
              head_dim=64, window=1000),
        # one new token of one sequence: latency
        _case("step_1", op="step", lengths="9001", q_heads=8),
        # one new token of 64 sequences, some shorter than the window, one slot of the batch unused
        _case("step_64", op="step", lengths="0,16211,15,9999,28174,21619,17691,4095,4096,4362,2547,7443,27028,21841,30103,4097,"
              "24*6001,24*1500", window=4096, n_sink=128),
        # a prompt with a state for each of 32 heads
        _case("linear_prompt_32k", op="linear", lengths="32768", kv_heads=32),
        # prompts and chunks that continue from states, single tokens among them, grouped narrow heads that forget slowly
        _case("linear_ragged_head_64", op="linear", lengths="12289,1,4500,7011,0,300,63,2050,1,1", q_heads=40, head_dim=64, decay=0.02),
        # one new token of one sequence: latency
        _case("state_1", op="state", lengths="1", q_heads=8),
        # one new token of 64 sequences
        _case("state_64", op="state", lengths="64*1", kv_heads=32),
        # 64 new tokens enter the cache
        _case("rotate_64", op="rotate", lengths="64*1", earlier="30*6001,33*1504,0"),
        # a prompt far into a long context enters the cache, wide layer
        _case("rotate_32k", op="rotate", lengths="32768", earlier="90000", q_heads=40),
        # a decode step of 64 sequences, every sixteenth of which needs a page
        _case("pages_64", op="pages", lengths="64*1", earlier="30*6001,30*1504,4*0"),
        # 700 requests arrive with prompts at once, others go on
        _case("pages_prompts", op="pages", lengths="700*180,300*1,200*25", earlier="700*0,300*901,200*16"),
    ]


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        top = most.setdefault(c["op"], {"bytes": 0, "flops": 0})
        top["bytes"], top["flops"] = max(top["bytes"], w["bytes"]), max(top["flops"], w["flops"])
    for _ in range(1000):
        op = rng.choice(["window", "window", "step", "linear", "linear", "state", "rotate", "pages"])
        heads = [(8, 8), (32, 8), (32, 8), (40, 8), (16, 4)] + ([(32, 32)] if op in ("linear", "state") else [])
        q_heads, kv_heads = rng.choice(heads)
        c = {**_DEFAULTS, "op": op, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": rng.choice([64, 128, 128, 128, 256]),
             "page": rng.choice([16, 16, 32, 64, 128, 7]), "window": int(round(math.exp(rng.uniform(0, math.log(6000))))),
             "n_sink": rng.choice([0, 1, 4, 64, 128]), "decay": rng.choice([1.0, 0.1, 0.02])}
        f32 = rng.random() < 0.15 and op not in ("step", "pages")
        if f32:
            c["dtype"], c["head_dim"] = "f32", rng.choice([64, 128])
        top_len = 8000 if f32 else 131072 if op == "step" else 40000
        total = int(round(math.exp(rng.uniform(math.log(20), math.log(top_len)))))
        n_seqs = 1 if rng.random() < 0.3 else rng.randint(2, 24)
        if op == "state":
            lengths = [1] * int(round(math.exp(rng.uniform(0, math.log(128)))))
        elif op == "pages":
            n_seqs = int(round(math.exp(rng.uniform(0, math.log(1500)))))
            lengths = [rng.choice([0, 1, 1, 1, rng.randint(1, 130)]) for _ in range(n_seqs)]
            c["spare"] = rng.choice([4, 4, 0, -3])       # pages short of what the step needs: not all are served
        else:
            cuts = sorted(rng.randint(1, max(1, total - 1)) for _ in range(n_seqs - 1))
            lengths = [b - a for a, b in zip([0] + cuts, cuts + [total]) if b > a]
        if op in ("window", "linear", "rotate") and rng.random() < 0.3:
            lengths = [rng.choice([0, 1, 1])] * rng.randint(1, 32) + lengths
        if op == "step" and rng.random() < 0.5:
            lengths = [max(0, n - rng.randint(0, 2)) for n in lengths]
        if op == "pages" or (op in ("window", "rotate") and rng.random() < 0.6):
            c["earlier"] = ",".join(str(int(math.exp(rng.uniform(0, math.log(3000 if op == "pages" else 30000)))) - 1) for _ in lengths)
        if op == "rotate":
            c["rot_dim"], c["norm"], c["pairs"] = c["head_dim"] // rng.choice([1, 1, 2]), rng.random() < 0.7, rng.random() < 0.3
        c["lengths"] = ",".join(str(n) for n in lengths)
        w, top = work(c), most[op]
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] and sum(_keys(c)) <= 400000 and sum(_numbers(c["lengths"])) > 0:
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


def _seen(first, last, window, n_sink):
    """Keys that the tokens at positions first .. last-1 see, in sum, and those that any of them sees."""
    p = np.arange(first, last, dtype=np.int64)
    low = np.maximum(p - window + 1, 0)
    pairs = int((p - low + 1 + np.minimum(low, n_sink)).sum())
    any_low = max(0, first - window + 1)
    return pairs, (last - any_low + min(any_low, n_sink)) if last > first else 0


def work(case):
    lengths, keys, d = _numbers(case["lengths"]), _keys(case), case["head_dim"]
    hq, hkv, e, op = case["q_heads"], case["kv_heads"], 4 if case["dtype"] == "f32" else 2, case["op"]
    tokens, seqs = sum(lengths), len(lengths)
    if op in ("window", "step"):
        new = [min(1, n) for n in lengths] if op == "step" else lengths
        seen = [_seen(k - n, k, case["window"], case["n_sink"]) for n, k in zip(new, keys)]
        return {"bytes": (seqs if op == "step" else tokens) * hq * (2 * d * e + 4) + 2 * sum(u for _, u in seen) * hkv * d * e,
                "flops": 4 * d * hq * sum(p for p, _ in seen)}
    if op in ("linear", "state"):
        # a token's product with the state, its own contribution to it; rows in and out, states in and out
        states = sum(2 if case["op"] == "state" or r % 3 == 1 else 1 for r in range(seqs))
        return {"bytes": tokens * (2 * hq + 2 * hkv) * d * e + states * hkv * d * d * 4, "flops": 2 * tokens * (hq + hkv) * d * d}
    if op == "rotate":
        return {"bytes": tokens * ((2 * hq + 4 * hkv) * d * e + 12), "flops": 0}
    new_pages = sum(-(-k // case["page"]) - -(-(k - n) // case["page"]) for n, k in zip(lengths, keys))
    return {"bytes": 12 * tokens + 8 * new_pages + 20 * seqs, "flops": 0}


# ---------------------------------------------------------------------------------------------------- inputs
def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _normal(gen, dtype, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _block_table(gen, lengths, page, width=0):
    """Pages of every sequence in random order, and how many there are."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(sum(need), generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros(len(lengths), max(need + [1, width]), dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, sum(need)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lengths = _numbers(case["lengths"])
    s = {**{k: case[k] for k in ("op", "q_heads", "kv_heads", "head_dim", "page", "window", "n_sink", "rot_dim", "norm", "pairs")},
         "lengths": lengths, "keys": _keys(case), "scale": 1.0 / math.sqrt(case["head_dim"]), "tokens": sum(lengths),
         "dtype": torch.float32 if case["dtype"] == "f32" else torch.bfloat16}
    {"window": _prepare_window, "step": _prepare_step, "linear": _prepare_linear, "state": _prepare_linear, "rotate": _prepare_rotate,
     "pages": _prepare_pages}[case["op"]](s, case, gen)
    return s


def _params(s, seqs, tokens):
    import paper_2605_06221_amd as up
    return up.make_params(num_seqs=seqs, total_tokens=tokens, block_size=64, num_q_heads=s["q_heads"], num_kv_heads=s["kv_heads"],
                          head_dim=s["head_dim"], qk_dtype=up.UP_F32 if s["dtype"] == torch.float32 else up.UP_BF16)


def _workspace(s, nbytes):
    s["ws_bytes"], s["ws"] = nbytes, torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")


def _prepare_window(s, case, gen):
    lengths, keys, dt = s["lengths"], s["keys"], s["dtype"]
    hkv, d, tokens = s["kv_heads"], s["head_dim"], s["tokens"]
    s["q"] = _normal(gen, dt, tokens, s["q_heads"], d)
    s["cu_host"], s["cu_k_host"] = _offsets(lengths), _offsets(keys)
    s["cu"], s["cu_k"] = torch.from_numpy(s["cu_host"]).cuda(), torch.from_numpy(s["cu_k_host"]).cuda()
    s["table"], rows = None, sum(keys)
    if case["earlier"]:
        s["table"], pages = _block_table(gen, keys, s["page"])
        rows = pages * s["page"]
    s["k"], s["v"] = _normal(gen, dt, rows, hkv, d), _normal(gen, dt, rows, hkv, d)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q_heads"], tokens, device="cuda")
    if own:
        import paper_2605_06221_amd as up
        s["p"] = _params(s, len(lengths), tokens)
        _workspace(s, up.uniprefill_attention_window_plan(s["p"], s["cu_host"], s["cu_k_host"] if case["earlier"] else None,
                                                          s["window"], s["n_sink"])[1])


def _prepare_step(s, case, gen):
    n_seqs = len(s["lengths"])
    s["table"], pages = _block_table(gen, s["lengths"], s["page"])
    s["q"] = _normal(gen, s["dtype"], n_seqs, s["q_heads"], s["head_dim"])
    s["k"] = _normal(gen, s["dtype"], pages * s["page"], s["kv_heads"], s["head_dim"])
    s["v"] = _normal(gen, s["dtype"], pages * s["page"], s["kv_heads"], s["head_dim"])
    s["kv_len"] = torch.tensor(s["lengths"], dtype=torch.int32, device="cuda")
    s["max_len"] = max(s["lengths"])
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(s["q_heads"], n_seqs, device="cuda")
    if own:
        import paper_2605_06221_amd as up
        s["p"] = _params(s, n_seqs, n_seqs)
        _workspace(s, up.uniprefill_attention_window_step_plan(s["p"], s["max_len"], s["window"], s["n_sink"])[1])


def _prepare_linear(s, case, gen):
    n_seqs, tokens, hkv, d, dt = len(s["lengths"]), s["tokens"], s["kv_heads"], s["head_dim"], s["dtype"]
    s["q"] = _normal(gen, dt, tokens, s["q_heads"], d)
    s["k"], s["v"] = _normal(gen, dt, tokens, hkv, d), _normal(gen, dt, tokens, hkv, d)
    # heads that forget within a token or two, to heads that remember hundreds (or ten thousands)
    s["log_decay"] = -case["decay"] * torch.exp2(-8.0 * torch.arange(1, hkv + 1, device="cuda") / hkv)
    s["cu_host"] = _offsets(s["lengths"])
    s["cu"] = torch.from_numpy(s["cu_host"]).cuda()
    # every sequence keeps its state in a slot of a pool; in a prompt's call one of three starts from the state in its slot, the others
    # from nothing
    slot = torch.randperm(n_seqs + 1, generator=gen, device="cuda")[:n_seqs].to(torch.int32)
    s["states"] = _normal(gen, torch.float32, n_seqs + 1, hkv, d, d)
    s["state_out"] = slot
    fresh = torch.arange(n_seqs, device="cuda") % 3 != 1
    s["state_in"] = slot if case["op"] == "state" else torch.where(fresh, torch.full_like(slot, -1), slot)
    s["out"] = torch.zeros_like(s["q"])
    if own:
        import paper_2605_06221_amd as up
        s["p"] = _params(s, n_seqs, tokens)
        if case["op"] == "linear":
            _workspace(s, up.uniprefill_linear_attention_plan(s["p"], s["cu_host"])[1])


def _prepare_rotate(s, case, gen):
    tokens, hq, hkv, d, dt = s["tokens"], s["q_heads"], s["kv_heads"], s["head_dim"], s["dtype"]
    # one row per token of a fused projection holds its queries, keys and values
    s["qkv"] = _normal(gen, dt, tokens, hq + 2 * hkv, d)
    s["q_weight"] = (1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(dt)
    s["k_weight"] = (1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(dt)
    s["inv_freq"] = (10000.0 ** (-torch.arange(0, s["rot_dim"], 2, dtype=torch.float64, device="cuda") / s["rot_dim"])).float()
    table, pages = _block_table(gen, s["keys"], s["page"])
    pos, slots = [], []
    for r, (n, k) in enumerate(zip(s["lengths"], s["keys"])):
        p = torch.arange(k - n, k, device="cuda")
        pos.append(p)
        slots.append(table[r].long()[p // s["page"]] * s["page"] + p % s["page"])
    s["pos"], s["slots"], s["num_slots"] = torch.cat(pos).to(torch.int32), torch.cat(slots), pages * s["page"]
    s["q_out"] = torch.zeros(tokens, hq, d, dtype=dt, device="cuda")
    s["k_cache"] = torch.zeros(s["num_slots"], hkv, d, dtype=dt, device="cuda")
    s["v_cache"] = torch.zeros_like(s["k_cache"])
    if own:
        import paper_2605_06221_amd as up
        row = (hq + 2 * hkv) * d
        s["p"] = up.make_params(num_seqs=len(s["lengths"]), total_tokens=tokens, block_size=64, num_q_heads=hq, num_kv_heads=hkv,
                                head_dim=d, q_row_stride=row, k_row_stride=row, qk_dtype=up.UP_F32 if dt == torch.float32 else up.UP_BF16)


def _prepare_pages(s, case, gen):
    keys, page, n_seqs = s["keys"], s["page"], len(s["lengths"])
    before = [k - n for k, n in zip(keys, s["lengths"])]
    width = max([-(-k // page) for k in keys]) + 2
    s["table"], used = _block_table(gen, before, page, width)
    need = sum(-(-k // page) - -(-b // page) for k, b in zip(keys, before))
    free = max(0, need + case["spare"])
    s["free"] = (used + torch.randperm(max(1, free), generator=gen, device="cuda")).to(torch.int32)
    s["num_free"] = torch.tensor([free], dtype=torch.int32, device="cuda")
    s["kv_len"] = torch.tensor(before, dtype=torch.int32, device="cuda")
    s["num_new"] = torch.tensor(s["lengths"], dtype=torch.int32, device="cuda")
    s["capacity"] = s["tokens"] + 8                     # a captured step is sized for somewhat more tokens than come
    s["slots"] = torch.zeros(s["capacity"], dtype=torch.int64, device="cuda")
    s["pos"] = torch.zeros(s["capacity"], dtype=torch.int32, device="cuda")
    s["cu"], s["cu_k"] = (torch.zeros(n_seqs + 1, dtype=torch.int32, device="cuda") for _ in range(2))
    s["new_len"], s["served"] = torch.zeros_like(s["kv_len"]), torch.zeros_like(s["num_free"])
    s["free_left"] = torch.zeros_like(s["num_free"])


# ---------------------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return {"window": _own_window, "step": _own_step, "linear": _own_linear, "state": _own_state, "rotate": _own_rotate,
                "pages": _own_pages}[s["op"]](s)
    return {"window": _plain_window, "step": _plain_step, "linear": _plain_linear, "state": _plain_state, "rotate": _plain_rotate,
            "pages": _plain_pages}[s["op"]](s)


def _own_window(s):
    import paper_2605_06221_amd as up
    hq, row, paged = s["q_heads"], s["kv_heads"] * s["head_dim"], s["table"] is not None
    up.uniprefill_attention_window(s["p"], s["q"], s["k"], s["v"], row, s["cu"], s["cu_host"], s["cu_k"] if paged else None,
                                   s["cu_k_host"] if paged else None, s["table"], s["table"].shape[1] if paged else 0, s["page"],
                                   s["window"], s["n_sink"], s["out"], hq * s["head_dim"], s["lse"], s["lse"].shape[1], s["ws"],
                                   s["ws_bytes"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_step(s):
    import paper_2605_06221_amd as up
    up.uniprefill_attention_window_step(s["p"], s["q"], s["k"], s["v"], s["kv_heads"] * s["head_dim"], s["kv_len"], s["max_len"],
                                        s["table"], s["table"].shape[1], s["page"], s["window"], s["n_sink"], s["out"],
                                        s["q_heads"] * s["head_dim"], s["lse"], s["lse"].shape[1], s["ws"], s["ws_bytes"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_linear(s):
    import paper_2605_06221_amd as up
    d = s["head_dim"]
    up.uniprefill_linear_attention(s["p"], s["q"], s["k"], s["v"], s["kv_heads"] * d, s["cu"], s["cu_host"], s["log_decay"],
                                   s["states"], s["kv_heads"] * d * d, s["states"].shape[0], s["state_in"], s["state_out"], s["out"],
                                   s["q_heads"] * d, s["ws"], s["ws_bytes"])
    return {"out": s["out"], "states": s["states"]}


def _own_state(s):
    import paper_2605_06221_amd as up
    d = s["head_dim"]
    up.uniprefill_linear_attention_step(s["p"], s["q"], s["k"], s["v"], s["kv_heads"] * d, s["log_decay"], s["states"],
                                        s["kv_heads"] * d * d, s["states"].shape[0], s["state_in"], s["state_out"], s["out"],
                                        s["q_heads"] * d)
    return {"out": s["out"], "states": s["states"]}


def _own_rotate(s):
    import paper_2605_06221_amd as up
    hq, hkv, d = s["q_heads"], s["kv_heads"], s["head_dim"]
    q, k, v = s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]
    up.uniprefill_norm_rotate(s["p"], q, k, v, (hq + 2 * hkv) * d, s["q_weight"] if s["norm"] else None,
                              s["k_weight"] if s["norm"] else None, 1e-6 if s["norm"] else 0.0, s["pos"], s["inv_freq"], s["rot_dim"],
                              s["pairs"], None, s["q_out"], hq * d, s["k_cache"], hkv * d, s["v_cache"], hkv * d, s["slots"],
                              s["num_slots"])
    return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"]}


def _own_pages(s):
    import paper_2605_06221_amd as up
    up.uniprefill_append_pages(s["kv_len"], s["num_new"], len(s["lengths"]), s["page"], s["table"], s["table"].shape[1], s["free"],
                               s["num_free"], s["free_left"], s["new_len"], s["cu"], s["cu_k"], s["pos"], s["slots"], s["capacity"],
                               s["served"])
    return _paged(s)


def _paged(s):
    return {k: s[k] for k in ("table", "free_left", "new_len", "cu", "cu_k", "pos", "slots", "served")}


def _blocks(s, size):
    """The sequences cut into pieces of `size` tokens: sequence, first token and packed rows of every piece, and which rows there are."""
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    count = (n + size - 1) // size
    total = sum(-(-m // size) for m in s["lengths"])
    r = torch.repeat_interleave(torch.arange(n.shape[0], device="cuda"), count, output_size=total)
    start = (torch.arange(total, device="cuda") - (torch.cumsum(count, 0) - count)[r]) * size
    token = start[:, None] + torch.arange(size, device="cuda")
    live = token < n[r][:, None]
    return r, start, (s["cu"][:-1].long()[r][:, None] + token).clamp(max=s["tokens"] - 1), live


def _attend(s, q, pos, key_row):
    """Queries q [b, rows, heads, d] in float at positions pos [b, rows] (ascending by one) over the keys that they see."""
    b, rows, hkv, d = q.shape[0], q.shape[1], s["kv_heads"], s["head_dim"]
    group, n_sink = s["q_heads"] // hkv, s["n_sink"]
    window = min(s["window"], max(s["keys"]) if s["op"] == "window" else s["max_len"])
    near = pos[:, :1] - (window - 1) + torch.arange(window + rows - 1, device="cuda")
    sinks = torch.arange(n_sink, device="cuda").expand(b, -1)
    see_near = (near[:, None] <= pos[:, :, None]) & (near[:, None] > pos[:, :, None] - window) & (near[:, None] >= n_sink)
    see = torch.cat([sinks[:, None] <= pos[:, :, None], see_near], 2)
    at = torch.cat([sinks, near], 1).clamp(min=0)
    at = key_row(torch.minimum(at, pos[:, -1:].clamp(min=0)))
    k = s["k"][at].float().permute(0, 2, 3, 1).contiguous()
    v = s["v"][at].float().permute(0, 2, 1, 3).contiguous()
    x = q.reshape(b, rows, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, rows * group, d)
    x = (torch.matmul(x, k) * s["scale"]).view(b, hkv, rows, group, -1)
    x.masked_fill_(~see[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top.clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(b, hkv, rows * group, -1), v).view(b, hkv, rows, group, d) / total.clamp(min=1e-30)
    lse = (top + torch.log(total)).squeeze(-1)
    return o.permute(0, 2, 1, 3, 4).reshape(b, rows, -1, d), lse.permute(1, 3, 0, 2).reshape(-1, b, rows)


def _plain_window(s):
    r, start, row, live = _blocks(s, 512)
    n, keys = (s["cu"][1:] - s["cu"][:-1]).long(), (s["cu_k"][1:] - s["cu_k"][:-1]).long()
    pos = (keys - n)[r][:, None] + start[:, None] + torch.arange(512, device="cuda")
    last = keys[r][:, None] - 1
    if s["table"] is None:
        def key_row(p):
            return s["cu_k"][:-1].long()[r][:, None] + torch.minimum(p, last)
    else:
        def key_row(p):
            p = torch.minimum(p, last)
            return s["table"][r[:, None], p // s["page"]].long() * s["page"] + p % s["page"]
    o, lse = _attend(s, s["q"][row].float(), pos, key_row)
    s["out"][row[live]] = o[live].to(s["out"].dtype)
    s["lse"][:, row[live]] = lse[:, live]
    return {"out": s["out"], "lse": s["lse"]}


def _plain_step(s):
    r = torch.arange(len(s["lengths"]), device="cuda")[:, None]
    pos = s["kv_len"].long()[:, None] - 1

    def key_row(p):
        return s["table"][r, p // s["page"]].long() * s["page"] + p % s["page"]
    o, lse = _attend(s, s["q"][:, None].float(), pos, key_row)
    s["out"].copy_(o[:, 0])
    s["lse"].copy_(lse[:, :, 0])
    return {"out": s["out"], "lse": s["lse"]}


def _start_states(s):
    given = s["state_in"] >= 0
    return torch.where(given[:, None, None, None], s["states"][s["state_in"].long().clamp(min=0)], torch.zeros((), device="cuda"))


def _plain_linear(s):
    size, hkv, d = 256, s["kv_heads"], s["head_dim"]
    group, ld = s["q_heads"] // hkv, s["log_decay"].double()
    r, start, row, live = _blocks(s, size)
    i, blocks, seqs = torch.arange(size, device="cuda"), r.shape[0], len(s["lengths"])
    q = (s["q"][row].float() * s["scale"]).view(blocks, size, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(blocks, hkv, group * size, d)
    k = (s["k"][row].float() * live[:, :, None, None]).permute(0, 2, 1, 3).contiguous()
    v = (s["v"][row].float() * live[:, :, None, None]).permute(0, 2, 1, 3).contiguous()
    # inside the pieces
    w = torch.where(i[:, None] >= i, torch.exp(ld[:, None, None] * (i[:, None] - i).clamp(min=0)), 0.0).float()
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(blocks, hkv, group, size, size).mul_(w[:, None])
    o = torch.matmul(x.view(blocks, hkv, group * size, size), v)
    # what every piece adds to the state; the state before every piece and after every sequence, all at once
    count = live.sum(1)
    w = torch.exp(ld[:, None] * (count[:, None, None] - 1 - i).clamp(min=0)).float()
    add = torch.matmul((k * w[..., None]).transpose(2, 3).contiguous(), v).permute(1, 0, 2, 3).reshape(hkv, blocks, d * d)
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    seq, when = torch.cat([r, torch.arange(seqs, device="cuda")]), torch.cat([start, n])
    apart = when[:, None] - (start + count)
    w = torch.where((seq[:, None] == r) & (apart >= 0), torch.exp(ld[:, None, None] * apart.clamp(min=0)), 0.0).float()
    first = _start_states(s).permute(1, 0, 2, 3).reshape(hkv, seqs, d * d)
    state = torch.matmul(w, add) + torch.exp(ld[:, None] * when).float()[..., None] * first[:, seq]
    before = state[:, :blocks].reshape(hkv, blocks, d, d).permute(1, 0, 2, 3).contiguous()
    w = torch.exp(ld[:, None] * (i + 1)).float()[:, None, :, None]
    o = o.view(blocks, hkv, group, size, d) + torch.matmul(q, before).view(blocks, hkv, group, size, d) * w
    s["out"][row[live]] = o.permute(0, 3, 1, 2, 4).reshape(blocks, size, -1, d)[live].to(s["out"].dtype)
    s["states"][s["state_out"].long()] = state[:, blocks:].reshape(hkv, seqs, d, d).permute(1, 0, 2, 3)
    return {"out": s["out"], "states": s["states"]}


def _plain_state(s):
    hkv, d, seqs = s["kv_heads"], s["head_dim"], len(s["lengths"])
    decay = torch.exp(s["log_decay"].double()).float()[:, None, None]
    state = _start_states(s) * decay + s["k"].float()[..., None] * s["v"].float()[:, :, None]
    o = torch.matmul((s["q"].float() * s["scale"]).view(seqs, hkv, -1, d), state)
    s["out"].copy_(o.view(seqs, -1, d))
    s["states"][s["state_out"].long()] = state
    return {"out": s["out"], "states": s["states"]}


def _plain_rotate(s):
    hq, hkv, rot = s["q_heads"], s["kv_heads"], s["rot_dim"]
    x = s["qkv"][:, :hq + hkv].float()
    if s["norm"]:
        weight = torch.cat([s["q_weight"].float().expand(hq, -1), s["k_weight"].float().expand(hkv, -1)])
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if s["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(2) if s["pairs"] else torch.cat([a, b], -1)
    x = torch.cat([turned, x[..., rot:]], -1).to(s["dtype"])
    s["q_out"].copy_(x[:, :hq])
    s["k_cache"][s["slots"]] = x[:, hq:]
    s["v_cache"][s["slots"]] = s["qkv"][:, hq + hkv:]
    return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"]}


def _plain_pages(s):
    page, table, free, most = s["page"], s["table"], s["free"], s["capacity"]
    had, new = s["kv_len"].long(), s["num_new"].long()
    old = (had + page - 1) // page
    need = (had + new + page - 1) // page - old
    fits = (torch.cumsum(need, 0) <= s["num_free"]) & (old + need <= table.shape[1]) & (torch.cumsum(new, 0) <= most)
    served = torch.cumprod(fits.long(), 0)
    need, new = need * served, new * served
    base = torch.cumsum(need, 0) - need
    # the free pages are taken from the list's end
    j = torch.arange(table.shape[1], device="cuda")
    at = (s["num_free"] - 1 - (base[:, None] + j - old[:, None])).clamp(0, free.shape[0] - 1)
    table.copy_(torch.where((j >= old[:, None]) & (j < (old + need)[:, None]), free[at], table))
    s["new_len"].copy_(had + new)
    s["cu"][1:], s["cu_k"][1:] = torch.cumsum(new, 0), torch.cumsum(had + new, 0)
    s["served"].copy_(served.sum())
    s["free_left"].copy_(s["num_free"] - need.sum())
    t = torch.arange(most, device="cuda")
    r = torch.searchsorted(s["cu"][1:].contiguous(), t.to(torch.int32), right=True).clamp(max=had.shape[0] - 1)
    p = had[r] + t - s["cu"][r]
    live = t < s["cu"][-1]
    s["pos"].copy_(torch.where(live, p, 0))
    s["slots"].copy_(torch.where(live, table[r, (p // page).clamp(0, table.shape[1] - 1)].long() * page + p % page, -1))
    return _paged(s)


# ---------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"window": _exact_window, "step": _exact_step, "linear": _exact_linear, "state": _exact_linear, "rotate": _exact_rotate,
            "pages": _exact_pages}[s["op"]](s)


def _pages_of(s, r, n):
    return (s["table"][r].long()[:, None] * s["page"] + torch.arange(s["page"], device="cuda")).reshape(-1)[:n]


def _exact_rows(s, q, first, rows):
    """Tokens q [n, heads, d] from position `first` on, over a sequence whose key i is row rows[i]."""
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[1], q.shape[0], dtype=torch.float64, device="cuda")
    for h in range(s["kv_heads"]):
        group = range(h * s["q_heads"] // s["kv_heads"], (h + 1) * s["q_heads"] // s["kv_heads"])
        k, v = s["k"][rows, h].double(), s["v"][rows, h].double()
        for a in range(0, q.shape[0], 2048):
            b = min(q.shape[0], a + 2048)
            pos = torch.arange(first + a, first + b, device="cuda")[:, None]
            low = max(0, first + a - s["window"] + 1)
            at = torch.cat([torch.arange(min(s["n_sink"], low), device="cuda"), torch.arange(low, first + b, device="cuda")])
            hidden = (at > pos) | ((pos - at >= s["window"]) & (at >= s["n_sink"]))
            for hq in group:
                x = torch.mm(q[a:b, hq].double(), k[at].T.contiguous()) * s["scale"]
                x[hidden] = -math.inf
                lse[hq, a:b] = torch.logsumexp(x, 1)
                out[a:b, hq] = torch.mm(torch.softmax(x, 1), v[at])
    return out, lse


def _exact_window(s):
    out, lse = [], []
    for r, (n, m) in enumerate(zip(s["lengths"], s["keys"])):
        a, b = int(s["cu_host"][r]), int(s["cu_k_host"][r])
        rows = torch.arange(b, b + m, device="cuda") if s["table"] is None else _pages_of(s, r, m)
        o, z = _exact_rows(s, s["q"][a:a + n], m - n, rows)
        out.append(o)
        lse.append(z)
    return {"out": torch.cat(out), "lse": torch.cat(lse, 1)}


def _exact_step(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for r, m in enumerate(s["lengths"]):
        if m:
            o, z = _exact_rows(s, s["q"][r:r + 1], m - 1, _pages_of(s, r, m))
            out[r], lse[:, r] = o[0], z[:, 0]
    return {"out": out, "lse": lse}


def _exact_linear(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    states = s["states"].double()
    for r, n in enumerate(s["lengths"]):
        a, source, to = int(s["cu_host"][r]), int(s["state_in"][r]), int(s["state_out"][r])
        for h in range(s["kv_heads"]):
            lam = math.exp(float(s["log_decay"][h]))
            state = s["states"][source, h].double() if source >= 0 else torch.zeros(s["head_dim"], s["head_dim"], dtype=torch.float64, device="cuda")
            k, v = s["k"][a:a + n, h].double(), s["v"][a:a + n, h].double()
            for lo in range(0, n, 1024):
                m = min(n, lo + 1024) - lo
                ages = torch.arange(m, dtype=torch.float64, device="cuda")
                seen = torch.tril(lam ** (ages[:, None] - ages).clamp(min=0))
                kc, vc = k[lo:lo + m], v[lo:lo + m]
                for hq in range(h * s["q_heads"] // s["kv_heads"], (h + 1) * s["q_heads"] // s["kv_heads"]):
                    q = s["q"][a + lo:a + lo + m, hq].double()
                    o = torch.mm(torch.mm(q, kc.T.contiguous()) * seen, vc) + torch.mm(q * (lam ** (ages + 1))[:, None], state)
                    out[a + lo:a + lo + m, hq] = o * s["scale"]
                state = lam ** m * state + torch.mm((kc * (lam ** (m - 1 - ages))[:, None]).T.contiguous(), vc)
            states[to, h] = state
    return {"out": out, "states": states}


def _exact_rotate(s):
    hq, hkv, rot = s["q_heads"], s["kv_heads"], s["rot_dim"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * s["inv_freq"].double())[:, None]

    def rotated(x, weight):
        x = x.double()
        if s["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + 1e-6) * weight.double()
        y = x.clone()
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if s["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., first], x[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y
    k, v = s["k_cache"].double(), s["v_cache"].double()
    k[s["slots"]] = rotated(s["qkv"][:, hq:hq + hkv], s["k_weight"])
    v[s["slots"]] = s["qkv"][:, hq + hkv:].double()
    return {"q": rotated(s["qkv"][:, :hq], s["q_weight"]), "k": k, "v": v}


def _exact_pages(s):
    table, free = s["table"].cpu().numpy().copy(), list(s["free"].cpu().numpy())[:int(s["num_free"])]
    new_len, cu, pos, slots, served, going = [], [0], [], [], 0, True
    for r, (n, k) in enumerate(zip(s["lengths"], s["keys"])):
        have = -(-(k - n) // s["page"])
        need = -(-k // s["page"]) - have
        going = going and need <= len(free) and have + need <= table.shape[1] and cu[-1] + n <= s["capacity"]
        if not going:
            n, k = 0, k - n
        else:
            served += 1
            for j in range(need):
                table[r, have + j] = free.pop()
        for p in range(k - n, k):
            pos.append(p)
            slots.append(int(table[r, p // s["page"]]) * s["page"] + p % s["page"])
        new_len.append(k)
        cu.append(cu[-1] + n)
    pad = s["capacity"] - len(pos)

    def ints(x, dtype=torch.int32):
        return torch.tensor(x, dtype=dtype, device="cuda")
    return {"table": ints(table), "free_left": ints([len(free)]), "new_len": ints(new_len), "cu": ints(cu),
            "cu_k": ints(_offsets(new_len)), "pos": ints(pos + [0] * pad), "slots": ints(slots + [-1] * pad, torch.int64),
            "served": ints([served])}
