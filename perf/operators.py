"""Timing cases of the serving operators: 8-bit quantisation by token, the 8-bit linear layer, and the 4-bit
key/value cache with the attention that reads it.

`run` computes a case in plain torch operations (fp32 throughout, one rounding at the end) or, with `own`
set, through the library's calls.  The formulas:

    quantise    a_b = max_n |x_bn|,  scale_b = a_b / 127,  q_bn = rint(x_bn * (127 / a_b))
    linear      y_bm = (sum_n q_bn W_mn) * scale_b * wscale_m + bias_m
    cache       per token, head and group of 32 values: step = fp16((hi - lo) / 15), base = fp16(lo),
                code = clamp(rint((x - base) / step), 0, 15); a code stands for code * step + base
    attention   out_i = sum_j softmax_j(scale * q_i . k_j) v_j over the positions j that query i may see

Sizes: the 4096-wide projections and 2048-token prompts of OPT-6.7B (32 heads of 128), the 12 heads of 64
and 128-token inputs of BERT-base, and ragged ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32            # values that share a step and a base in the cache
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one prompt's hidden states before a projection
        {"name": "quantise-prompt", "op": "quantise", "rows": 2048, "cols": 4096, "pad": 0, "dtype": "bf16"},
        # fp32 activations of a ragged batch, rows that are a slice of wider ones
        {"name": "quantise-odd", "op": "quantise", "rows": 333, "cols": 1001, "pad": 23, "dtype": "f32"},
        # a projection for one generated token
        {"name": "linear-token", "op": "linear", "B": 1, "N": 4096, "M": 4096, "dtype": "bf16", "bias": True},
        # the fused query/key/value projection of a prompt
        {"name": "linear-prompt", "op": "linear", "B": 2048, "N": 4096, "M": 12288, "dtype": "bf16", "bias": True},
        # activations that arrive in 8 bits with their scales, no size a multiple of anything, fp32 result
        {"name": "linear-odd", "op": "linear", "B": 197, "N": 1001, "M": 770, "dtype": "i8", "bias": True},
        # one new token for each of 64 sequences
        {"name": "append-tokens", "op": "append", "seqs": 64, "kv_heads": 8, "dim": 128, "page": 16, "new": 1,
         "history": 1500, "dtype": "bf16"},
        # the keys and values of three prompts of different lengths
        {"name": "append-prompts", "op": "append", "seqs": 3, "kv_heads": 32, "dim": 128, "page": 64, "new": 2048,
         "history": 0, "dtype": "bf16"},
        # the smallest call: one token over a short context, narrow heads
        {"name": "decode-short", "op": "attend", "seqs": 1, "heads": 12, "kv_heads": 12, "dim": 64, "page": 16, "new": 1,
         "history": 509, "causal": True, "window": 0},
        # a serving batch: 32 sequences of different lengths, shared key/value heads
        {"name": "decode-batch", "op": "attend", "seqs": 32, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "new": 1,
         "history": 8191, "causal": True, "window": 0},
        # one very long context
        {"name": "decode-long", "op": "attend", "seqs": 1, "heads": 32, "kv_heads": 8, "dim": 128, "page": 256, "new": 1,
         "history": 100002, "causal": True, "window": 0},
        # a whole prompt, every head with its own keys
        {"name": "prompt", "op": "attend", "seqs": 1, "heads": 32, "kv_heads": 32, "dim": 128, "page": 64, "new": 2048,
         "history": 0, "causal": True, "window": 0},
        # pieces of prompts behind earlier context, a sliding window, lengths that end inside pages and tiles
        {"name": "pieces-window", "op": "attend", "seqs": 7, "heads": 16, "kv_heads": 4, "dim": 64, "page": 32, "new": 509,
         "history": 1533, "causal": True, "window": 1000},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantise", "linear", "linear", "append", "attend", "attend", "attend"])
    if op == "quantise":
        rows = _log(rng, 1, 4096)
        return {"op": op, "rows": rows, "cols": _log(rng, 64, min(16384, (1 << 24) // rows)), "pad": rng.choice([0, 0, 8, 23]),
                "dtype": rng.choice(["bf16", "f32"])}
    if op == "linear":
        B, N = _log(rng, 1, 2048), _log(rng, 64, 16384)
        return {"op": op, "B": B, "N": N, "M": _log(rng, 64, min(16384, 2048 * 4096 * 12288 // (B * N))),
                "dtype": rng.choice(["bf16", "f32", "i8"]), "bias": rng.random() < 0.5}
    kv_heads, dim, page = rng.choice([1, 2, 4, 8, 12, 32]), rng.choice([64, 128]), rng.choice([16, 32, 64, 256])
    seqs = _log(rng, 1, 64)
    if op == "append":
        new = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, min(2048, (1 << 23) // (seqs * kv_heads * dim))))
        return {"op": op, "seqs": seqs, "kv_heads": kv_heads, "dim": dim, "page": page, "new": new, "history": _log(rng, 1, 1500),
                "dtype": rng.choice(["bf16", "f32"])}
    group = rng.choice([1, 1, 2, 4, 8])
    heads = min(64, kv_heads * group) // kv_heads * kv_heads
    room = (1 << 27) // (seqs * kv_heads * dim)                    # cached positions a sequence
    if rng.random() < 0.5:
        new = 1
    else:
        new = _log(rng, 2, max(2, min(2048, room // 2, int(math.sqrt((1 << 27) / (seqs * heads))))))
    most = max(1, min(60000, room - new, (1 << 27) // (seqs * heads * new) - new))
    return {"op": op, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "new": new,
            "history": _log(rng, 1, most), "causal": rng.random() < 0.8, "window": rng.choice([0, 0, 0, _log(rng, 16, 4096)])}


# ---- sizes of a batch of sequences ------------------------------------------------------------------------------


def _lengths(case):
    """(new tokens, positions in the cache with them) of each sequence: fixed by the case, no two alike."""
    S = case["seqs"]
    new = [max(1, case["new"] * ((3 * s + 1) % S + 1) // S) for s in range(S)]
    return new, [case["history"] * ((5 * s + 2) % S + 1) // S + n for s, n in enumerate(new)]


def _visible(case):
    """(pairs of a query and a position it sees, positions that any query sees) over all sequences."""
    pairs = seen = 0
    for n, length in zip(*_lengths(case)):
        at = range(length - n, length)
        top = [p + 1 if case["causal"] else length for p in at]
        low = [max(0, p + 1 - case["window"]) if case["window"] else 0 for p in at]
        pairs += sum(t - w for t, w in zip(top, low))
        seen += max(top) - min(low)
    return pairs, seen


def work(case):
    size = {"f32": 4, "bf16": 2, "i8": 1}.get(case.get("dtype"), 2)
    if case["op"] == "quantise":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size + 1) + n * (1 + 4) + 8 * case["rows"], "flops": 3 * n}
    if case["op"] == "linear":
        B, N, M = case["B"], case["N"], case["M"]
        return {"bytes": B * N * size + N * M + B * M * (2 if case["dtype"] == "bf16" else 4) + 4 * M, "flops": 2 * B * N * M}
    D, Hkv = case["dim"], case["kv_heads"]
    packed = 2 * Hkv * (D // 2 + D // GROUP * 4)                   # bytes of one position: codes, steps and bases
    if case["op"] == "append":
        n = sum(_lengths(case)[0])
        return {"bytes": n * (2 * Hkv * D * (size + 4) + 2 * packed), "flops": 8 * n * Hkv * D}
    n, (pairs, seen) = sum(_lengths(case)[0]), _visible(case)
    return {"bytes": seen * packed + 4 * n * case["heads"] * D, "flops": 4 * pairs * case["heads"] * D}


# ---- inputs -----------------------------------------------------------------------------------------------------


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _activations(gen, rows, cols):
    """Hidden states: normal values, one channel in 100 about ten times larger."""
    loud = 1 + 9 * (torch.rand(cols, generator=gen, device="cuda") < 0.01).float()
    return _normal(gen, rows, cols) * loud


def _keys_values(gen, tokens, heads, dim, dtype):
    """Keys carry an offset of their own in each channel, values do not."""
    k = _normal(gen, tokens, heads, dim) + 2 * _normal(gen, 1, heads, dim)
    return k.to(dtype), _normal(gen, tokens, heads, dim).to(dtype)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "quantise":
        x = _activations(gen, case["rows"], case["cols"] + case["pad"]).to(DTYPES[case["dtype"]])
        return {"x": x[:, :case["cols"]]}
    if case["op"] == "linear":
        w = _normal(gen, case["M"], case["N"]) * 0.02
        w8, w_scale = _quantise(w)
        got = {"w8": w8.to(torch.int8), "w_scale": w_scale, "bias": 0.1 * _normal(gen, case["M"]) if case["bias"] else None}
        x = _activations(gen, case["B"], case["N"])
        if case["dtype"] == "i8":
            x8, got["x_scale"] = _quantise(x)
            return {**got, "x": x8.to(torch.int8)}
        return {**got, "x": x.to(DTYPES[case["dtype"]])}
    new, length = _lengths(case)
    S, H, D, page = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    per_seq = -(-max(length) // page)
    got = {"table": torch.randperm(S * per_seq, generator=gen, device="cuda").to(torch.int32).view(S, per_seq),
           "seq_len": torch.tensor(length, dtype=torch.int32, device="cuda"),
           "q_start": torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)}
    if case["op"] == "append":
        got["k"], got["v"] = _keys_values(gen, sum(new), H, D, DTYPES[case["dtype"]])
        return got
    # the cached keys and values, every page filled to its end: what lies behind a sequence's length is stale
    got["k"], got["v"] = _keys_values(gen, S * per_seq * page, H, D, torch.bfloat16)
    got["q"] = _normal(gen, sum(new), case["heads"], D).to(torch.bfloat16)
    return got


def prepare(case, seed):
    got = _inputs(case, seed)
    state = {"case": case, **got}
    if own:
        import paper_2308_07641_b200 as lib
        state["lib"] = lib
    if case["op"] == "linear":
        if own:
            state["layer"] = lib.Int8Linear(got["w8"], got["w_scale"], got["bias"])
            state["layer"].reserve(case["B"], case["dtype"])
    if case["op"] in ("append", "attend"):
        S, per_seq = got["table"].shape
        if own:
            state["cache"] = lib.KV4Cache(case["kv_heads"], case["dim"], n_pages=S * per_seq, page_tokens=case["page"])
        else:
            state["pool"] = _empty_pool(S * per_seq, case)
        if case["op"] == "attend":
            full = torch.full((S,), per_seq * case["page"], dtype=torch.int32, device="cuda")
            start = torch.arange(S + 1, dtype=torch.int32, device="cuda") * (per_seq * case["page"])
            if own:
                state["cache"].append(got["k"], got["v"], got["table"], full, start)
            else:
                _append(state["pool"], got["k"], got["v"], got["table"], full, start, case["page"])
            del state["k"], state["v"]
    return state


# ---- the operators in plain form ----------------------------------------------------------------------------------


def _quantise(x):
    x = x.float()
    a = x.abs().amax(dim=1)
    q = torch.round(x * torch.where(a > 0, 127.0 / a, torch.zeros_like(a))[:, None])
    return q, a / 127.0


def _linear(state):
    x = state["x"]
    if x.dtype == torch.int8:
        q, scale = x.float(), state["x_scale"]
    else:
        q, scale = _quantise(x)
    y = (q @ state["w8"].float().t()) * scale[:, None] * state["w_scale"][None, :]
    if state["bias"] is not None:
        y = y + state["bias"]
    return y.to(torch.bfloat16) if x.dtype == torch.bfloat16 else y


def _empty_pool(n_pages, case):
    shape = (n_pages, case["page"], case["kv_heads"])
    groups = case["dim"] // GROUP
    make = lambda last, dtype: torch.zeros(shape + (last,), dtype=dtype, device="cuda")  # noqa: E731
    return {**{name + "_codes": make(case["dim"] // 2, torch.uint8) for name in "kv"},
            **{name + "_step": make(groups, torch.float16) for name in "kv"},
            **{name + "_base": make(groups, torch.float16) for name in "kv"}}


def _places(table, seq_len, q_start, n, page):
    """Where the new tokens' positions lie: page numbers and places in the page."""
    new = q_start[1:] - q_start[:-1]
    seq = torch.repeat_interleave(torch.arange(len(seq_len), device=table.device), new, output_size=n)
    at = torch.arange(n, device=table.device) - q_start[seq] + (seq_len - new)[seq]
    return table[seq, at // page].long(), at % page


def _append(pool, k, v, table, seq_len, q_start, page):
    where = _places(table, seq_len, q_start, k.shape[0], page)
    for name, x in (("k", k), ("v", v)):
        g = x.float().unflatten(-1, (-1, GROUP))
        lo, hi = g.amin(-1).clamp(-65000, 65000), g.amax(-1).clamp(-65000, 65000)
        step, base = ((hi - lo) / 15).half(), lo.half()
        s = step.float()
        code = torch.round((g - base.float()[..., None]) * torch.where(s > 0, 1 / s, torch.zeros_like(s))[..., None])
        code = code.clamp(0, 15).to(torch.uint8).flatten(-2)
        pool[name + "_codes"][where] = code[..., 0::2] | (code[..., 1::2] << 4)
        pool[name + "_step"][where] = step
        pool[name + "_base"][where] = base


def _values(pool, name, where):
    packed = pool[name + "_codes"][where]
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    return (code * pool[name + "_step"][where].float()[..., None] + pool[name + "_base"][where].float()[..., None]).flatten(-2)


def _attend(state):
    case, table, seq_len, q_start = state["case"], state["table"].long(), state["seq_len"].long(), state["q_start"].long()
    page, H, D = case["page"], case["kv_heads"], case["dim"]
    new, length = _lengths(case)
    S, max_q, max_kv, G = len(new), max(new), max(length), case["heads"] // case["kv_heads"]
    at = torch.arange(max_kv, device="cuda")
    where = (table[:, at // page], (at % page).expand(S, max_kv))
    k = _values(state["pool"], "k", where).permute(0, 2, 1, 3)                                   # [S, H, max_kv, D]
    v = _values(state["pool"], "v", where).permute(0, 2, 1, 3)
    i = torch.arange(max_q, device="cuda")
    n_new = q_start[1:] - q_start[:-1]
    row = (q_start[:-1, None] + i).clamp(max=state["q"].shape[0] - 1)                             # [S, max_q]
    q = state["q"][row].float().unflatten(2, (H, G)).permute(0, 2, 1, 3, 4).reshape(S, H, max_q * G, D)
    scores = (q @ k.transpose(-1, -2)).mul_(1 / math.sqrt(D)).view(S, H, max_q, G, max_kv)
    pos = (seq_len - n_new)[:, None] + i
    hide = at >= seq_len[:, None, None]
    if case["causal"]:
        hide = hide | (at > pos[..., None])
    if case["window"]:
        hide = hide | (at <= pos[..., None] - case["window"])
    scores.masked_fill_(hide[:, None, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    e = scores.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    out = (e.view(S, H, max_q * G, max_kv) @ v).view(S, H, max_q, G, D) / torch.where(total > 0, total, torch.ones_like(total))
    out = out.permute(0, 2, 1, 3, 4).reshape(S, max_q, H * G, D)
    return out[i < n_new[:, None]].to(torch.bfloat16)


def run(state):
    case = state["case"]
    if case["op"] == "quantise":
        if own:
            return state["lib"].dequantize(*state["lib"].quantize(state["x"]))
        q, scale = _quantise(state["x"])
        return q * scale[:, None]
    if case["op"] == "linear":
        if own:
            return state["layer"](state["x"], state.get("x_scale"))
        return _linear(state)
    table, seq_len, q_start = state["table"], state["seq_len"], state["q_start"]
    if case["op"] == "append":
        n = state["k"].shape[0]
        if own:
            state["cache"].append(state["k"], state["v"], table, seq_len, q_start)
            return state["cache"].read(n, table, seq_len, q_start)
        _append(state["pool"], state["k"], state["v"], table, seq_len, q_start, case["page"])
        where = _places(table, seq_len, q_start, n, case["page"])
        return _values(state["pool"], "k", where), _values(state["pool"], "v", where)
    if own:
        new, length = _lengths(case)
        return state["cache"].attend(state["q"], table, seq_len, q_start, max_q=max(new), max_kv=max(length),
                                     causal=case["causal"], window=case["window"])
    return _attend(state)


# ---- the operators from their definitions, in 64 bits ---------------------------------------------------------------


def _exact_cached(x):
    """What a [..., D] tensor of keys or values stands for once it is in the cache.  Which code a number gets is
    defined in fp32; what the code stands for is taken in 64 bits."""
    d = x.float().reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    lowest = d.min(-1, keepdim=True).values
    step = ((d.max(-1, keepdim=True).values - lowest) / 15).to(torch.float16)
    base = lowest.to(torch.float16)
    code = ((d - base.float()) * step.float().reciprocal()).round().clamp(0, 15).nan_to_num(0.0)
    return (base.double() + code.double() * step.double()).reshape(x.shape)


def _exact_rows(x):
    """The same for a row in 8 bits."""
    top = x.float().abs().max(1, keepdim=True).values
    return (x.float() * (127 / top)).round().double() * (top.double() / 127)


def exact(case, seed):
    got = _inputs(case, seed)
    if case["op"] == "quantise":
        return _exact_rows(got["x"])
    if case["op"] == "linear":
        if case["dtype"] == "i8":
            x = got["x"].double() * got["x_scale"].double()[:, None]
        else:
            x = _exact_rows(got["x"])
        y = torch.nn.functional.linear(x, got["w8"].double() * got["w_scale"].double()[:, None])
        return y if got["bias"] is None else y + got["bias"].double()
    if case["op"] == "append":
        return _exact_cached(got["k"]), _exact_cached(got["v"])
    new, length = _lengths(case)
    G, D, room = case["heads"] // case["kv_heads"], case["dim"], got["k"].shape[0] // len(new)
    outs, first = [], 0
    for s, (n, size) in enumerate(zip(new, length)):
        q = got["q"][first:first + n].double()
        j, p = torch.arange(size, device="cuda")[None, :], torch.arange(size - n, size, device="cuda")[:, None]
        seen = (j <= p) if case["causal"] else (j >= 0).expand(n, size)
        if case["window"]:
            seen = seen & (j > p - case["window"])
        heads = []
        for h in range(case["heads"]):
            k = _exact_cached(got["k"][s * room:s * room + size, h // G])
            v = _exact_cached(got["v"][s * room:s * room + size, h // G])
            logits = torch.where(seen, (q[:, h] @ k.T) / math.sqrt(D), torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            heads.append(torch.softmax(logits, dim=1) @ v)
        outs.append(torch.stack(heads, 1))
        first += n
    return torch.cat(outs)
