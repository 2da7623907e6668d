"""The serving operators together, as examples/serving_layer.py runs them: a decoder layer on ragged prompts and then token by
token, against the same layer in plain 64-bit operations on the same (quantised) weights and cache."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2308_07641_b200 import build
    build.build()
    spec = importlib.util.spec_from_file_location("serving_layer", os.path.join(ROOT, "examples", "serving_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _rows8(x):
    """Rows through 8 bits and back."""
    import torch
    a = x.abs().amax(dim=1, keepdim=True)
    return torch.round(x / a * 127) * (a / 127)


class Plain:
    """The layer in 64 bits, intermediates rounded to bf16 where the layer hands them on in bf16; the attention over what the
    layer's own cache holds (a number that falls the other way there is off by a fifteenth of its group's range, and what the
    cache makes of its input is tested by itself)."""

    def __init__(self, weights, heads, kv_heads):
        import torch
        self.w = {k: _rows8(weights[k].double()) for k in ("qkv", "out")}
        self.t = {k: [torch.from_numpy(np.asarray(m, dtype=np.float64)).cuda() for m in weights[k]] for k in ("up", "down")}
        self.heads, self.kv_heads, self.width = heads, kv_heads, weights["out"].shape[0]

    def ternary(self, name, x):
        U, S, V = self.t[name]
        return ((x @ V.T) * S) @ U.T

    def forward(self, x, new, cached):
        import torch
        r = lambda t: t.float().bfloat16().double()  # noqa: E731
        norm = lambda t: r(torch.nn.functional.layer_norm(t, (self.width,)))  # noqa: E731
        d, G = self.width // self.heads, self.heads // self.kv_heads
        qkv = r(_rows8(norm(x)) @ self.w["qkv"].T)
        q, k, v = qkv.split([self.heads * d, self.kv_heads * d, self.kv_heads * d], dim=1)
        outs, first = [], 0
        for s, n in enumerate(new):
            rows = slice(first, first + n)
            first += n
            K, V = cached[s]
            L = K.shape[0]
            for have, t in ((K, k), (V, v)):       # the new positions are there: each within a step of what went in
                t = t[rows].unflatten(1, (self.kv_heads, d))
                g = t.unflatten(-1, (-1, 32))
                step = ((g.amax(-1, keepdim=True) - g.amin(-1, keepdim=True)) / 15).expand_as(g).flatten(-2)
                assert ((have[L - n:] - t).abs() <= 1.6 * step + 0.02 * t.abs()).all()
            K, V = (t.repeat_interleave(G, dim=1) for t in (K, V))
            score = torch.einsum("ihd,jhd->hij", q[rows].unflatten(1, (self.heads, d)), K) / d ** 0.5
            see = torch.arange(L, device="cuda")[None, :] <= torch.arange(L - n, L, device="cuda")[:, None]
            p = torch.softmax(score.masked_fill(~see, -torch.inf), dim=-1)
            outs.append(torch.einsum("hij,jhd->ihd", p, V).flatten(1))
        x = r(x + r(_rows8(r(torch.cat(outs))) @ self.w["out"].T))
        return r(x + r(self.ternary("down", torch.relu(r(self.ternary("up", norm(x)))))))


@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (8, 2, 128)])
def test_layer_prompts_then_tokens(example, heads, kv_heads, dim):
    """Both sides round to bf16 and to 8 bits at the same places, from numbers that differ by bf16 roundings: an 8-bit value
    that falls the other way is off by 2^-7 of its row's largest, a bf16 one by 2^-8 of itself.  A row of the result passes
    about ten such steps, each at most 2^-8 of its size in the 2-norm, independent: below 2^-6 together."""
    import torch
    width = heads * dim
    weights = example.random_weights(width, heads, kv_heads, 2 * width, width, seed=heads)
    new = [70, 1, 33, 128]
    table, n_pages = example.pages([n + 4 for n in new], 16)
    layer = example.ServedLayer(weights, heads, kv_heads, n_pages, 16)
    layer.reserve(sum(new))
    plain = Plain(weights, heads, kv_heads)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.randn(sum(new), width, generator=gen, device="cuda").to(torch.bfloat16)
    start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    seq_len = torch.tensor(new, dtype=torch.int32, device="cuda")
    y = layer.forward(x, table, seq_len, start, max(new))

    def cached():
        """What the cache holds of each sequence."""
        lens = seq_len.tolist()
        at = torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")
        k, v = layer.cache.read(sum(lens), table, seq_len, at)
        return list(zip(k.double().split(lens), v.double().split(lens)))

    def check(got, want):
        off = (got.double() - want).norm(dim=1) / want.norm(dim=1)
        assert off.max() <= 2.0 ** -6, f"worst row is {float(off.max()):.3g} off"

    check(y, plain.forward(x.double(), new, cached()))
    for step in range(3):
        seq_len += 1
        x = torch.randn(len(new), width, generator=gen, device="cuda").to(torch.bfloat16)
        y = layer.forward(x, table, seq_len)
        check(y, plain.forward(x.double(), [1] * len(new), cached()))
    assert layer.status() == 0


def test_example_runs(example, monkeypatch, capsys):
    import sys
    monkeypatch.setattr(sys, "argv", ["serving_layer.py", "--width", "512", "--heads", "8", "--kv-heads", "4", "--ffn", "1024", "--rank", "512",
                                      "--sequences", "3", "--prompt", "90", "--tokens", "4"])
    example.main()
    assert "a token" in capsys.readouterr().out
