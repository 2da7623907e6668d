"""Timing cases of a served decoder layer's operators beside its products: the root-mean-square norm that adds the residual
and hands on 8-bit rows, low-rank adapters of many requests beside a shared projection, the append to the 4-bit cache with the
position rotation on the way, and attention over that cache with a sliding window and a few first positions that stay visible.

`run` computes a case in plain torch operations (fp32, rounded once at the end) or, with `own` set, through the library's
calls.  The formulas:

    norm        h = round(x + residual) to x's type;  rho_b = 1 / sqrt(mean_n h_bn^2 + eps);  y_bn = h_bn rho_b w_n
                in 8 bits: t_bn = h_bn w_n in fp32, a_b = max_n |t_bn|, q_bn = rint(t_bn ((1 / a_b) 127)),
                scale_b = rho_b a_b / 127
    adapters    y_b = base_b + c_s B_s (A_s x_b) with s the adapter of row b's sequence, or y_b = base_b without one
    rotation    pairs (u, v) of a head, rotated by the angle of their position: (u cos - v sin, v cos + u sin), in fp32;
                keys and values then go into the cache (4 bits, groups of 32), queries are rounded to their type
    attention   out_i = sum_j p_ij v_j, p_i = softmax(scale q_i . k_j) over j <= P_i with j > P_i - window or j < sinks

Sizes: widths of 4096 and 12288, prompts of 2048 tokens and 32 heads of 128 (OPT-6.7B), 12 heads of 64 (BERT-base), and ragged
ones around them.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 32            # values that share a step and a base in the cache
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the residual stream of a few generated tokens, on its way to an 8-bit projection
        {"name": "norm-tokens", "op": "norm", "rows": 8, "cols": 4096, "pad": 0, "dtype": "bf16", "residual": True, "bits8": True},
        # the same of a whole prompt
        {"name": "norm-prompt", "op": "norm", "rows": 2048, "cols": 4096, "pad": 0, "dtype": "bf16", "residual": True, "bits8": True},
        # the last norm of a ragged batch, in fp32, rows that are a slice of wider ones
        {"name": "norm-odd", "op": "norm", "rows": 333, "cols": 1001, "pad": 23, "dtype": "f32", "residual": False, "bits8": False},
        # one token for each of 64 requests, most with an adapter of their own, beside the fused query/key/value projection
        {"name": "adapt-tokens", "op": "adapt", "seqs": 64, "new": 1, "slots": 48, "rank": 16, "N": 4096, "M": 12288, "dtype": "bf16"},
        # prompts of five requests
        {"name": "adapt-prompts", "op": "adapt", "seqs": 5, "new": 682, "slots": 8, "rank": 64, "N": 4096, "M": 12288, "dtype": "bf16"},
        # rows that arrive in 8 bits with their scales, no size a multiple of anything, fp32 results
        {"name": "adapt-odd", "op": "adapt", "seqs": 7, "new": 49, "slots": 5, "rank": 9, "N": 1001, "M": 770, "dtype": "i8"},
        # one new token for each of 64 sequences
        {"name": "rotate-tokens", "op": "rotate", "seqs": 64, "heads": 32, "kv_heads": 8, "dim": 128, "turned": 128, "interleaved": False,
         "page": 16, "new": 1, "history": 1500, "dtype": "bf16"},
        # three prompts of different lengths, every head with its own keys
        {"name": "rotate-prompts", "op": "rotate", "seqs": 3, "heads": 32, "kv_heads": 32, "dim": 128, "turned": 128,
         "interleaved": False, "page": 64, "new": 2048, "history": 0, "dtype": "bf16"},
        # pieces far behind in long contexts, fp32, half of each head turned, neighbours as pairs
        {"name": "rotate-far", "op": "rotate", "seqs": 2, "heads": 12, "kv_heads": 12, "dim": 64, "turned": 32, "interleaved": True,
         "page": 32, "new": 77, "history": 130000, "dtype": "f32"},
        # a serving batch behind long contexts of which a window and the first positions are read
        {"name": "sinks-tokens", "op": "attend", "seqs": 32, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "new": 1,
         "history": 20000, "causal": True, "window": 4096, "sinks": 4},
        # a long prompt with a window a quarter as long
        {"name": "sinks-prompt", "op": "attend", "seqs": 1, "heads": 32, "kv_heads": 32, "dim": 128, "page": 64, "new": 4096,
         "history": 0, "causal": True, "window": 1024, "sinks": 16},
        # pieces of prompts behind earlier context; first positions, window and lengths end inside pages and tiles
        {"name": "sinks-pieces", "op": "attend", "seqs": 7, "heads": 16, "kv_heads": 4, "dim": 64, "page": 32, "new": 509,
         "history": 3533, "causal": True, "window": 777, "sinks": 131},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "adapt", "adapt", "adapt", "rotate", "rotate", "attend", "attend", "attend"])
    if op == "norm":
        rows = _log(rng, 1, 4096)
        return {"op": op, "rows": rows, "cols": _log(rng, 64, min(16384, (1 << 23) // rows)), "pad": rng.choice([0, 0, 8, 23]),
                "dtype": rng.choice(["bf16", "f32"]), "residual": rng.random() < 0.6, "bits8": rng.random() < 0.6}
    if op == "adapt":
        seqs, new = _log(rng, 1, 128), 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
        seqs = max(1, min(seqs, 4096 // new))
        N = _log(rng, 64, min(12288, (1 << 24) // (seqs * new)))
        return {"op": op, "seqs": seqs, "new": new, "slots": rng.choice([1, 4, 16, 64]), "rank": rng.choice([4, 8, 9, 16, 32, 64]),
                "N": N, "M": _log(rng, 64, min(12288, (1 << 24) // (seqs * new))), "dtype": rng.choice(["bf16", "bf16", "f32", "i8"])}
    kv_heads, dim, page = rng.choice([1, 2, 4, 8, 12, 32]), rng.choice([64, 128]), rng.choice([16, 32, 64, 256])
    heads = min(64, kv_heads * rng.choice([1, 1, 2, 4, 8])) // kv_heads * kv_heads
    seqs = _log(rng, 1, 64)
    if op == "rotate":
        new = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, min(2048, (1 << 22) // (seqs * heads * dim))))
        return {"op": op, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "turned": rng.choice([dim, dim, dim // 2, 24]),
                "interleaved": rng.random() < 0.3, "page": page, "new": new, "history": _log(rng, 1, 130000), "dtype": rng.choice(["bf16", "f32"])}
    room = (1 << 27) // (seqs * kv_heads * dim)                    # cached positions a sequence
    if rng.random() < 0.5:
        new = 1
    else:
        new = _log(rng, 2, max(2, min(2048, room // 2, int(math.sqrt((1 << 27) / (seqs * heads))))))
    most = max(1, min(60000, room - new, (1 << 27) // (seqs * heads * new) - new))
    return {"op": op, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "new": new, "history": _log(rng, 1, most),
            "causal": rng.random() < 0.8, "window": _log(rng, 16, 4096), "sinks": rng.choice([1, 4, 4, 16, _log(rng, 2, 300)])}


# ---- sizes of a batch of sequences ------------------------------------------------------------------------------


def _lengths(case):
    """(new tokens, positions in the cache with them) of each sequence: fixed by the case, no two alike."""
    S = case["seqs"]
    new = [max(1, case["new"] * ((3 * s + 1) % S + 1) // S) for s in range(S)]
    return new, [case.get("history", 0) * ((5 * s + 2) % S + 1) // S + n for s, n in enumerate(new)]


def _visible(case):
    """(pairs of a query and a position it sees, positions that any query sees) over all sequences."""
    pairs = seen = 0
    for n, length in zip(*_lengths(case)):
        at = range(length - n, length)
        top = [p + 1 if case["causal"] else length for p in at]
        low = [max(0, p + 1 - case["window"]) for p in at]
        first = [min(w, case["sinks"], t) for w, t in zip(low, top)]
        pairs += sum(t - w + f for t, w, f in zip(top, low, first))
        seen += max(top) - min(low) + min(min(low), case["sinks"])
    return pairs, seen


def _ranks(case):
    """Ranks of the adapters: the case's, half and a quarter of it."""
    return [max(1, case["rank"] >> (s % 3)) for s in range(case["slots"])]


def _requests(case, seed):
    """The adapter of each sequence: some are asked for often, one request in eight has none (-1)."""
    gen = torch.Generator()
    gen.manual_seed(seed)
    often = (torch.rand(case["seqs"], generator=gen).pow(1.5) * case["slots"]).long().clamp(max=case["slots"] - 1)
    return torch.where(torch.rand(case["seqs"], generator=gen) < 0.125, -1, often).tolist()


def work(case):
    size = {"f32": 4, "bf16": 2, "i8": 1}.get(case.get("dtype"), 2)
    if case["op"] == "norm":
        n = case["rows"] * case["cols"]
        rows = n * size * (3 if case["residual"] else 1) + 4 * case["cols"]
        # in 8 bits and back to numbers, or numbers at once
        return {"bytes": rows + (n * (1 + 1 + 4) + 8 * case["rows"] if case["bits8"] else n * size), "flops": 5 * n}
    if case["op"] == "adapt":
        out = 2 if case["dtype"] == "bf16" else 4
        n, N, M = sum(_lengths(case)[0]), case["N"], case["M"]
        # weights: as many adapters as requests may ask for; the seed says which
        ranks = sorted(_ranks(case), reverse=True)[:case["seqs"]]
        return {"bytes": n * N * size + 2 * n * M * out + 2 * sum(ranks) * (N + M), "flops": 2 * n * (N + M) * sum(ranks) // len(ranks)}
    D, H, Hkv = case["dim"], case["heads"], case["kv_heads"]
    packed = 2 * Hkv * (D // 2 + D // GROUP * 4)                   # bytes of one position: codes, steps and bases
    n = sum(_lengths(case)[0])
    if case["op"] == "rotate":
        return {"bytes": n * (2 * H * D * size + 2 * Hkv * D * (size + 4) + 2 * packed + 4 * case["turned"]), "flops": 8 * n * (H + Hkv) * D}
    pairs, seen = _visible(case)
    return {"bytes": seen * packed + 4 * n * H * D, "flops": 4 * pairs * H * D}


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


def _angles(positions, turned):
    """cos and sin of each position's angles, side by side: computed in 64 bits, kept in fp32."""
    rate = 10000.0 ** (-torch.arange(0, turned, 2, dtype=torch.float64, device="cuda") / turned)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * rate
    return torch.cat((a.cos(), a.sin()), 1).float()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "norm":
        rows, cols, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
        x = _activations(gen, rows, cols + case["pad"]).to(dtype)[:, :cols]
        r = (3 * _normal(gen, rows, cols + case["pad"])).to(dtype)[:, :cols] if case["residual"] else None
        return {"x": x, "residual": r, "weight": 1 + 0.2 * _normal(gen, cols)}
    new, length = _lengths(case)
    start = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    if case["op"] == "adapt":
        n, N, M = sum(new), case["N"], case["M"]
        asked = _requests(case, seed)
        got = {"asked": asked, "slots": torch.tensor(asked, dtype=torch.int32, device="cuda"), "q_start": start,
               "A": [(_normal(gen, r, N) / math.sqrt(N)).to(torch.bfloat16) for r in _ranks(case)],
               "B": [(_normal(gen, M, r) / math.sqrt(r)).to(torch.bfloat16) for r in _ranks(case)],
               "scale": [0.25 * (1 + s % 4) for s in range(case["slots"])], "x_scale": None}
        x = _activations(gen, n, N)
        if case["dtype"] == "i8":
            a = x.abs().amax(1)
            got["x"], got["x_scale"] = torch.round(x * (127 / a)[:, None]).to(torch.int8), a / 127
        else:
            got["x"] = x.to(DTYPES[case["dtype"]])
        got["base"] = _normal(gen, n, M).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        return got
    S, H, D, page = case["seqs"], case["kv_heads"], case["dim"], case["page"]
    got = {"seq_len": torch.tensor(length, dtype=torch.int32, device="cuda"), "q_start": start}
    if case["op"] == "rotate":
        # pages for the new positions in any order; earlier ones are one shared page, which the call does not touch
        first = [(size - n) // page for n, size in zip(new, length)]
        need = [-(-size // page) - f for f, size in zip(first, length)]
        numbers = 1 + torch.randperm(sum(need), generator=gen, device="cuda").to(torch.int32)
        got["table"] = torch.zeros(S, max(f + m for f, m in zip(first, need)), dtype=torch.int32, device="cuda")
        for s, part in enumerate(numbers.split(need)):
            got["table"][s, first[s]:first[s] + need[s]] = part
        got["pages"] = 1 + sum(need)
        got["k"], got["v"] = _keys_values(gen, sum(new), H, D, DTYPES[case["dtype"]])
        got["q"] = _normal(gen, sum(new), case["heads"], D).to(DTYPES[case["dtype"]])
        got["angles"] = _angles(max(length), case["turned"])
        return got
    per_seq = -(-max(length) // page)
    got["table"] = torch.randperm(S * per_seq, generator=gen, device="cuda").to(torch.int32).view(S, per_seq)
    got["pages"] = S * per_seq
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
    if case["op"] == "adapt":
        if own:
            state["adapters"] = lib.LowRankAdapters(case["N"], case["M"], max_rank=case["rank"], n_slots=case["slots"])
            for s in range(case["slots"]):
                state["adapters"].set(s, got["A"][s], got["B"][s], got["scale"][s])
            state["adapters"].reserve(got["x"].shape[0])
            del state["A"], state["B"]
        else:
            state["A"] = [a.float() for a in got["A"]]
            state["B"] = [b.float() for b in got["B"]]
            if case["new"] == 1:                                   # one row each: adapters side by side, padded to one rank
                pad = lambda m, dim: torch.cat((m, m.new_zeros([case["rank"] - m.shape[d] if d == dim else m.shape[d] for d in (0, 1)])), dim)  # noqa: E731
                state["A"] = torch.stack([pad(a, 0) for a in state["A"]])
                state["B"] = torch.stack([pad(b, 1) for b in state["B"]])
                state["scales"] = torch.tensor(got["scale"] + [0.0], device="cuda")
    if case["op"] in ("rotate", "attend"):
        if own:
            state["cache"] = lib.KV4Cache(case["kv_heads"], case["dim"], n_pages=got["pages"], page_tokens=case["page"])
        else:
            state["pool"] = _empty_pool(got["pages"], case)
    if case["op"] == "attend":
        S, per_seq = got["table"].shape
        full = torch.full((S,), per_seq * case["page"], dtype=torch.int32, device="cuda")
        start = torch.arange(S + 1, dtype=torch.int32, device="cuda") * (per_seq * case["page"])
        if own:
            state["cache"].append(got["k"], got["v"], got["table"], full, start)
        else:
            _append(state["pool"], got["k"].float(), got["v"].float(), _places(got["table"], full, start, got["k"].shape[0], case["page"]))
        del state["k"], state["v"]
    return state


# ---- the operators in plain form ----------------------------------------------------------------------------------


def _norm(state):
    x, w, case = state["x"], state["weight"], state["case"]
    h = x
    if case["residual"]:
        h = (x.float() + state["residual"].float()).to(x.dtype)
    f = h.float()
    rho = 1 / torch.sqrt((f * f).mean(1) + EPS)
    if case["bits8"]:
        t = f * w
        a = t.abs().amax(1)
        q = torch.round(t * torch.where(a > 0, (1 / a) * 127, torch.zeros_like(a))[:, None])
        y = q * (a * (1 / 127) * rho)[:, None]
    else:
        y = (f * rho[:, None] * w).to(x.dtype)
    return (y, h) if case["residual"] else y


def _adapt(state):
    x = state["x"].float()
    if state["x_scale"] is not None:
        x = x * state["x_scale"][:, None]
    y = state["base"].float()
    if state["case"]["new"] == 1:
        at = state["slots"].long()
        z = torch.bmm(state["A"][at.clamp(min=0)], x[:, :, None]) * state["scales"][at][:, None, None]
        y = y + torch.bmm(state["B"][at.clamp(min=0)], z)[:, :, 0]
    else:
        y, first = y.clone(), 0
        for s, n in zip(state["asked"], _lengths(state["case"])[0]):
            if s >= 0:
                y[first:first + n] += (x[first:first + n] @ state["A"][s].t()) @ state["B"][s].t() * state["scale"][s]
            first += n
    return y.to(state["base"].dtype)


def _empty_pool(n_pages, case):
    shape = (n_pages, case["page"], case["kv_heads"])
    groups = case["dim"] // GROUP
    make = lambda last, dtype: torch.zeros(shape + (last,), dtype=dtype, device="cuda")  # noqa: E731
    return {**{name + "_codes": make(case["dim"] // 2, torch.uint8) for name in "kv"},
            **{name + "_step": make(groups, torch.float16) for name in "kv"},
            **{name + "_base": make(groups, torch.float16) for name in "kv"}}


def _positions(seq_len, q_start, n):
    """Sequence and position of each of the n new rows."""
    new = q_start[1:] - q_start[:-1]
    seq = torch.repeat_interleave(torch.arange(len(seq_len), device=seq_len.device), new, output_size=n)
    return seq, torch.arange(n, device=seq_len.device) - q_start[seq] + (seq_len - new)[seq]


def _places(table, seq_len, q_start, n, page):
    """Where the new tokens' positions lie: page numbers and places in the page."""
    seq, at = _positions(seq_len, q_start, n)
    return table[seq, at // page].long(), at % page


def _append(pool, k, v, where):
    for name, x in (("k", k), ("v", v)):
        g = x.unflatten(-1, (-1, GROUP))
        lo, hi = g.amin(-1).clamp(-65000, 65000), g.amax(-1).clamp(-65000, 65000)
        step, base = ((hi - lo) * (1 / 15)).half(), lo.half()
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


def _turn(x, angles, interleaved):
    """x [rows, heads, dim] in fp32, the first numbers of each head rotated; angles [rows, turned]: cos, then sin."""
    turned = angles.shape[1]
    c, s = angles[:, None, :turned // 2], angles[:, None, turned // 2:]
    part, rest = x[..., :turned], x[..., turned:]
    if interleaved:
        u, v = part[..., 0::2], part[..., 1::2]
        part = torch.stack((u * c - v * s, v * c + u * s), -1).flatten(-2)
    else:
        u, v = part[..., :turned // 2], part[..., turned // 2:]
        part = torch.cat((u * c - v * s, v * c + u * s), -1)
    return torch.cat((part, rest), -1)


def _rotate(state):
    case, n = state["case"], state["k"].shape[0]
    angles = state["angles"][_positions(state["seq_len"], state["q_start"], n)[1]]
    where = _places(state["table"], state["seq_len"], state["q_start"], n, case["page"])
    _append(state["pool"], _turn(state["k"].float(), angles, case["interleaved"]), state["v"].float(), where)
    q = _turn(state["q"].float(), angles, case["interleaved"]).to(state["q"].dtype)
    return q, _values(state["pool"], "k", where), _values(state["pool"], "v", where)


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
    hide = (at <= pos[..., None] - case["window"]) & (at >= case["sinks"])
    hide = hide | (at >= seq_len[:, None, None])
    if case["causal"]:
        hide = hide | (at > pos[..., None])
    scores.masked_fill_(hide[:, None, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True).clamp_min(-3e38)
    e = scores.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    out = (e.view(S, H, max_q * G, max_kv) @ v).view(S, H, max_q, G, D) / torch.where(total > 0, total, torch.ones_like(total))
    out = out.permute(0, 2, 1, 3, 4).reshape(S, max_q, H * G, D)
    return out[i < n_new[:, None]].to(torch.bfloat16)


def run(state):
    case = state["case"]
    if case["op"] == "norm":
        if not own:
            return _norm(state)
        lib, x, w, r = state["lib"], state["x"], state["weight"], state["residual"]
        if not case["bits8"]:
            return lib.rms_norm(x, w, EPS, residual=r)
        if case["residual"]:
            q, scale, h = lib.rms_norm_quantize(x, w, EPS, residual=r)
            return lib.dequantize(q, scale), h
        return lib.dequantize(*lib.rms_norm_quantize(x, w, EPS))
    if case["op"] == "adapt":
        if own:
            return state["adapters"](state["x"], state["base"], state["slots"], state["q_start"], x_scale=state["x_scale"])
        return _adapt(state)
    table, seq_len, q_start = state["table"], state["seq_len"], state["q_start"]
    if case["op"] == "rotate":
        if own:
            q = state["cache"].append_rotated(state["q"], state["k"], state["v"], state["angles"], table, seq_len, q_start,
                                              interleaved=case["interleaved"])
            return (q, *state["cache"].read(state["k"].shape[0], table, seq_len, q_start))
        return _rotate(state)
    if own:
        new, length = _lengths(case)
        return state["cache"].attend(state["q"], table, seq_len, q_start, max_q=max(new), max_kv=max(length), causal=case["causal"],
                                     window=case["window"], sinks=case["sinks"])
    return _attend(state)


# ---- the operators from their definitions, in 64 bits ---------------------------------------------------------------


def _exact_cached(x):
    """What a [..., D] tensor of keys or values stands for once it is in the cache.  Which code a number gets is
    defined in fp32; what the code stands for is taken in 64 bits."""
    d = x.float().reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    lowest = d.min(-1, keepdim=True).values
    step = ((d.max(-1, keepdim=True).values - lowest) * torch.tensor(1 / 15, device=x.device)).to(torch.float16)
    base = lowest.to(torch.float16)
    code = ((d - base.float()) * step.float().reciprocal()).round().clamp(0, 15).nan_to_num(0.0)
    return (base.double() + code.double() * step.double()).reshape(x.shape)


def _exact_turned(x, angles, interleaved):
    """Each number of the rotated heads by itself, in the type of x and angles."""
    half = angles.shape[1] // 2
    out = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
        cos, sin = angles[:, None, i], angles[:, None, half + i]
        out[..., a] = x[..., a] * cos - x[..., b] * sin
        out[..., b] = x[..., b] * cos + x[..., a] * sin
    return out


def exact(case, seed):
    got = _inputs(case, seed)
    if case["op"] == "norm":
        h = got["x"] if got["residual"] is None else (got["x"].double() + got["residual"].double()).to(got["x"].dtype)
        d, w = h.double(), got["weight"].double()
        size = (d.square().sum(1, keepdim=True) / case["cols"] + EPS).sqrt()
        if case["bits8"]:                                          # which of the 255 steps is defined in fp32
            t = h.float().mul(got["weight"])
            top = t.abs().max(1, keepdim=True).values
            y = t.mul(top.reciprocal().mul(127)).round().double() * (top.double() / 127 / size)
        else:
            y = d / size * w
        return y if got["residual"] is None else (y, h.double())
    new, length = _lengths(case)
    if case["op"] == "adapt":
        rows = torch.arange(case["seqs"], device="cuda").repeat_interleave(torch.tensor(new, device="cuda"))
        mine = got["slots"].long()[rows]
        x = got["x"].double()
        if got["x_scale"] is not None:
            x = x * got["x_scale"].double()[:, None]
        y = got["base"].double()
        for s in sorted(set(got["asked"]) - {-1}):
            y[mine == s] += got["scale"][s] * torch.linalg.multi_dot([x[mine == s], got["A"][s].double().T, got["B"][s].double().T])
        return y
    if case["op"] == "rotate":
        at = torch.cat([torch.arange(size - n, size, device="cuda") for n, size in zip(new, length)])
        angles = got["angles"][at]
        q = _exact_turned(got["q"].double(), angles.double(), case["interleaved"])
        return q, _exact_cached(_exact_turned(got["k"].float(), angles, case["interleaved"])), _exact_cached(got["v"])
    G, D, room = case["heads"] // case["kv_heads"], case["dim"], got["k"].shape[0] // len(new)
    outs, first = [], 0
    for s, (n, size) in enumerate(zip(new, length)):
        q = got["q"][first:first + n].double()
        j, p = torch.arange(size, device="cuda")[None, :], torch.arange(size - n, size, device="cuda")[:, None]
        seen = (p - j < case["window"]) | (j < case["sinks"])
        if case["causal"]:
            seen = seen & (j <= p)
        heads = []
        for h in range(case["heads"]):
            k = _exact_cached(got["k"][s * room:s * room + size, h // G])
            v = _exact_cached(got["v"][s * room:s * room + size, h // G])
            logits = torch.where(seen, (q[:, h] @ k.T) / math.sqrt(D), torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
            heads.append(torch.softmax(logits, dim=1) @ v)
        outs.append(torch.stack(heads, 1))
        first += n
    return torch.cat(outs)
