"""The norms, adapters, rotated append and windowed attention together, as examples/serving_layer.py runs them: a decoder layer on
ragged prompts and then token by token, in the eager form and as a replayed graph, against the same layer in plain 64-bit operations
on the same (quantised) weights and cache."""
import os

import numpy as np
import pytest

from tests.test_serving_layer_gpu import ROOT, _rows8, example  # noqa: F401

pytestmark = pytest.mark.gpu


class Plain:
    """The layer in 64 bits, intermediates rounded where the layer hands them on in bf16 or 8 bits; the attention over what the
    layer's own cache holds (what the cache makes of its input is tested by itself)."""

    def __init__(self, weights, adapters, heads, kv_heads, window, sinks):
        import torch
        self.w = {k: _rows8(weights[k].double()) for k in ("qkv", "out")}
        self.t = {k: [torch.from_numpy(np.asarray(m, dtype=np.float64)).cuda() for m in weights[k]] for k in ("up", "down")}
        self.norm = [weights["norm1"].double(), weights["norm2"].double()]
        self.adapters = [[(A.double(), B.double(), c) for A, B, c in pair] for pair in adapters]
        self.heads, self.kv_heads, self.width, self.window, self.sinks = heads, kv_heads, weights["out"].shape[0], window, sinks

    def adapt(self, which, x, y, asked, new):
        import torch
        out, first = [], 0
        for s, n in zip(asked, new):
            part = y[first:first + n]
            if s >= 0:
                A, B, c = self.adapters[s][which]
                part = part + c * (x[first:first + n] @ A.T) @ B.T
            out.append(part)
            first += n
        return torch.cat(out)

    def turned(self, x, at):
        """x [rows, heads, d] at positions at."""
        import torch
        half = x.shape[-1] // 2
        a = at.double()[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        c, s = a.cos()[:, None], a.sin()[:, None]
        u, v = x[..., :half], x[..., half:]
        return torch.cat((u * c - v * s, v * c + u * s), -1)

    def forward(self, x, stream, asked, new, cached):
        import torch
        r = lambda t: t.float().bfloat16().double()  # noqa: E731
        rho = lambda t: 1 / (t.square().mean(1, keepdim=True) + 1e-6).sqrt()  # noqa: E731
        d, G = self.width // self.heads, self.heads // self.kv_heads
        stream = r(x + stream)
        x8 = _rows8(stream * rho(stream) * self.norm[0])
        qkv = r(self.adapt(0, x8, r(x8 @ self.w["qkv"].T), asked, new))
        q, k, v = (t.unflatten(1, (-1, d)) for t in qkv.split([self.heads * d, self.kv_heads * d, self.kv_heads * d], dim=1))
        at = torch.cat([torch.arange(c[0].shape[0] - n, c[0].shape[0], device="cuda") for c, n in zip(cached, new)])
        q, k = r(self.turned(q, at)), self.turned(k, at)
        outs, first = [], 0
        for n, (K, V) in zip(new, cached):
            rows, L = slice(first, first + n), K.shape[0]
            first += n
            for have, t in ((K, k[rows]), (V, v[rows])):       # the new positions are there: each within a step of what went in
                g = t.unflatten(-1, (-1, 32))
                step = ((g.amax(-1, keepdim=True) - g.amin(-1, keepdim=True)) / 15).expand_as(g).flatten(-2)
                assert ((have[L - n:] - t).abs() <= 1.6 * step + 0.02 * t.abs()).all()
            K, V = (t.repeat_interleave(G, dim=1) for t in (K, V))
            score = torch.einsum("ihd,jhd->hij", q[rows], K) / d ** 0.5
            j, p = torch.arange(L, device="cuda")[None, :], torch.arange(L - n, L, device="cuda")[:, None]
            see = (j <= p) & ((j > p - self.window) | (j < self.sinks))
            outs.append(torch.einsum("hij,jhd->ihd", torch.softmax(score.masked_fill(~see, -torch.inf), dim=-1), V).flatten(1))
        a = r(torch.cat(outs))
        y = r(self.adapt(1, a, r(_rows8(a) @ self.w["out"].T), asked, new))
        stream = r(y + stream)
        y = r(stream * rho(stream) * self.norm[1])
        for name in ("up", "down"):
            U, S, V = self.t[name]
            y = r(((y @ V.T) * S) @ U.T)
            if name == "up":
                y = torch.relu(y)
        return y, stream


@pytest.mark.parametrize("heads,kv_heads,dim,window,sinks", [(4, 4, 64, 40, 3), (8, 2, 128, 70, 17)])
def test_layer_prompts_then_tokens(example, heads, kv_heads, dim, window, sinks):  # noqa: F811
    """Both sides round to bf16 and to 8 bits at the same places, from numbers that differ by such roundings: an 8-bit value that
    falls the other way is off by 2^-7 of its row's largest, a bf16 one by 2^-8 of itself.  A row of the result passes about
    fourteen such steps, each at most 2^-8 of its size in the 2-norm, independent: below 2^-6 together (14^(1/2) < 4)."""
    import torch
    width, rank = heads * dim, 9
    weights = example.random_weights(width, heads, kv_heads, 2 * width, width, seed=heads)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    adapters = [(example.random_adapter((heads + 2 * kv_heads) * dim, width, rank, gen), example.random_adapter(width, width, rank, gen))
                for _ in range(3)]
    new, asked = [70, 1, 33, 128], [2, 0, -1, 2]
    table, n_pages = example.pages([n + 6 for n in new], 16)
    layer = example.AdaptedLayer(weights, heads, kv_heads, n_pages, 16, n_adapters=4, adapter_rank=16, positions=200, window=window, sinks=sinks)
    for i, (qkv, out) in enumerate(adapters):
        layer.set_adapter(i, qkv, out)
    layer.reserve(sum(new))
    plain = Plain(weights, adapters, heads, kv_heads, window, sinks)
    draw = lambda n: torch.randn(n, width, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    seq_len = torch.tensor(new, dtype=torch.int32, device="cuda")
    slots = torch.tensor(asked, dtype=torch.int32, device="cuda")

    def cached():
        """What the cache holds of each sequence."""
        lens = seq_len.tolist()
        at = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
        k, v = layer.cache.read(sum(lens), table, seq_len, at)
        return list(zip(k.double().split(lens), v.double().split(lens)))

    def check(got, want):
        for g, w in zip(got, want):
            off = (g.double() - w).norm(dim=1) / w.norm(dim=1)
            assert off.max() <= 2.0 ** -6, f"worst row is {float(off.max()):.3g} off"

    x, stream = draw(sum(new)), draw(sum(new))
    check(layer.forward(x, stream, slots, table, seq_len, start, max(new)), plain.forward(x.double(), stream.double(), asked, new, cached()))
    x, stream = draw(4), draw(4)
    seq_len += 1
    check(layer.forward(x, stream, slots, table, seq_len), plain.forward(x.double(), stream.double(), asked, [1] * 4, cached()))
    # the same step as a graph: other rows, lengths and adapters each time
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out = layer.forward(x, stream, slots, table, seq_len)
    for step in range(3):
        x.copy_(draw(4))
        stream.copy_(draw(4))
        asked = [step, -1, (step + 1) % 3, 3]                    # (slot 3 is empty)
        slots.copy_(torch.tensor(asked))
        seq_len += 1
        graph.replay()
        asked[3] = -1
        check(out, plain.forward(x.double(), stream.double(), asked, [1] * 4, cached()))
    assert layer.status() == 0


def test_example_runs_with_adapters(example, monkeypatch, capsys):  # noqa: F811
    import sys
    monkeypatch.setattr(sys, "argv", ["serving_layer.py", "--width", "512", "--heads", "8", "--kv-heads", "4", "--ffn", "1024", "--rank", "512",
                                      "--sequences", "3", "--prompt", "90", "--tokens", "4", "--adapters", "2", "--window", "50", "--sinks", "4"])
    example.main()
    assert "a token" in capsys.readouterr().out
    assert os.path.exists(os.path.join(ROOT, "examples", "serving_layer.py"))
