"""A decoder layer as it is served: ternary feed-forward layers (TSVDLinear), dense projections in 8 bits (Int8Linear) and
attention over a key/value cache in 4 bits (KV4Cache).  Random weights; sizes of one OPT-6.7B layer unless told otherwise.
With --adapters the layer is of a later kind: root-mean-square norms that add the residual, one of them straight into 8-bit rows,
low-rank adapters of each sequence beside the projections, positions by rotation, a sliding window with visible first positions.

    python examples/serving_layer.py [--width 4096 --heads 32 --ffn 16384 --rank 4096 --sequences 8 --prompt 512 --tokens 32]
    python examples/serving_layer.py --adapters 8 [--adapter-rank 16 --window 1024 --sinks 4]

Runs a batch of prompts of different lengths, then generates one token after another (hidden states, no vocabulary), and prints
the time of each.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2308_07641_b200 import (Int8Linear, KV4Cache, LowRankAdapters, TSVDLinear, quantize, rms_norm, rms_norm_quantize,  # noqa: E402
                                   rotary_table)
from paper_2308_07641_b200.binding import TSVD_FLAG_OUT_BF16  # noqa: E402


class ServedLayer:
    """x + out(attention(norm(x))), then that + down(relu(up(norm(.)))).  `weights` holds the dense matrices as float tensors
    [out, in] ("qkv", "out") and the ternary ones as triples of arrays (U, S, V) ("up", "down")."""

    def __init__(self, weights: dict, heads: int, kv_heads: int, n_pages: int, page_tokens: int = 64):
        self.width = weights["out"].shape[0]
        self.heads, self.kv_heads, self.dim = heads, kv_heads, self.width // heads
        self.qkv = Int8Linear(*quantize(weights["qkv"]))
        self.out = Int8Linear(*quantize(weights["out"]))
        self.up, self.down = TSVDLinear(*weights["up"]), TSVDLinear(*weights["down"])
        self.cache = KV4Cache(kv_heads, self.dim, n_pages, page_tokens)

    def reserve(self, rows: int) -> None:
        """Scratch for calls of up to that many rows, so that none of them allocates."""
        for layer in (self.qkv, self.out, self.up, self.down):
            layer.reserve(rows, "bf16")

    def forward(self, x, page_table, seq_len, q_start=None, max_q=None):
        """x: bfloat16 [rows, width], the rows of the sequences one after another (q_start; one each where None); seq_len and
        page_table as KV4Cache takes them, the rows included."""
        norm = torch.nn.functional.layer_norm
        rows, d = x.shape[0], self.dim
        qkv = self.qkv(norm(x, (self.width,)))
        # q, k and v are slices of one projection's rows: read where they lie
        q = qkv[:, :self.heads * d].unflatten(1, (self.heads, d))
        k, v = (qkv[:, (self.heads + i * self.kv_heads) * d:(self.heads + (i + 1) * self.kv_heads) * d].unflatten(1, (self.kv_heads, d))
                for i in range(2))
        self.cache.append(k, v, page_table, seq_len, q_start)
        a = self.cache.attend(q, page_table, seq_len, q_start, max_q=max_q)
        x = x + self.out(a.view(rows, self.width))
        return x + self.down(torch.relu(self.up(norm(x, (self.width,)))))

    def status(self) -> int:
        """The first status word that is not zero (see include/tsvd_serving.h)."""
        return self.cache.status() or self.qkv.status() or self.out.status()


class AdaptedLayer(ServedLayer):
    """A layer that hands its sums on: it takes the stream h and what the layer before adds to it, and returns what it adds itself
    with the stream.  `weights` holds the norms as well ("norm1", "norm2", float32 [width]); adapters are set by number."""

    def __init__(self, weights: dict, heads: int, kv_heads: int, n_pages: int, page_tokens: int = 64, n_adapters: int = 8,
                 adapter_rank: int = 16, positions: int = 4096, window: int = 0, sinks: int = 0):
        super().__init__(weights, heads, kv_heads, n_pages, page_tokens)
        self.norm1, self.norm2 = weights["norm1"], weights["norm2"]
        self.adapt_qkv = LowRankAdapters(self.width, weights["qkv"].shape[0], adapter_rank, n_adapters)
        self.adapt_out = LowRankAdapters(self.width, self.width, adapter_rank, n_adapters)
        self.rotary = rotary_table(positions, self.dim)
        self.window, self.sinks = window, sinks

    def set_adapter(self, number: int, qkv, out) -> None:
        """Triples (A [rank, in], B [out, rank], factor) beside the two dense projections."""
        self.adapt_qkv.set(number, *qkv)
        self.adapt_out.set(number, *out)

    def reserve(self, rows: int) -> None:
        super().reserve(rows)
        self.qkv.reserve(rows, "i8")
        self.adapt_qkv.reserve(rows)
        self.adapt_out.reserve(rows)

    def forward(self, x, stream, adapters, page_table, seq_len, q_start=None, max_q=None):
        """x, stream: bfloat16 [rows, width]; adapters: int32 [sequences], -1 for none; the rest as ServedLayer takes it.  Returns
        (x, stream) for the layer behind it."""
        rows, d = x.shape[0], self.dim
        x8, scale, stream = rms_norm_quantize(x, self.norm1, residual=stream)
        qkv = self.qkv(x8, scale, flags=TSVD_FLAG_OUT_BF16)
        self.adapt_qkv(x8, qkv, adapters, q_start, x_scale=scale, out=qkv)
        q = qkv[:, :self.heads * d].unflatten(1, (self.heads, d))
        k, v = (qkv[:, (self.heads + i * self.kv_heads) * d:(self.heads + (i + 1) * self.kv_heads) * d].unflatten(1, (self.kv_heads, d))
                for i in range(2))
        q = self.cache.append_rotated(q, k, v, self.rotary, page_table, seq_len, q_start)
        a = self.cache.attend(q, page_table, seq_len, q_start, max_q=max_q, window=self.window, sinks=self.sinks).view(rows, self.width)
        y = self.out(a)
        self.adapt_out(a, y, adapters, q_start, out=y)
        y, stream = rms_norm(y, self.norm2, residual=stream)
        return self.down(torch.relu(self.up(y))), stream

    def status(self) -> int:
        return super().status() or self.adapt_qkv.status() or self.adapt_out.status()


def ternary(rng, out: int, inner: int, rank: int, density: float = 0.25):
    """U [out, rank], S [rank], V [rank, inner] whose product keeps the size of its input."""
    draw = lambda *s: (rng.integers(0, 2, s, dtype=np.int8) * 2 - 1) * (rng.random(s, dtype=np.float32) < density)  # noqa: E731
    S = np.exp(0.3 * rng.standard_normal(rank)) / (density * np.sqrt(inner * rank))
    return draw(out, rank).astype(np.int8), S.astype(np.float32), draw(rank, inner).astype(np.int8)


def random_weights(width: int, heads: int, kv_heads: int, ffn: int, rank: int, seed: int = 0) -> dict:
    gen, rng = torch.Generator(device="cuda"), np.random.default_rng(seed)
    gen.manual_seed(seed)
    dense = lambda o, i: torch.randn(o, i, generator=gen, device="cuda") / i ** 0.5  # noqa: E731
    return {"qkv": dense((heads + 2 * kv_heads) * (width // heads), width), "out": dense(width, width),
            "up": ternary(rng, ffn, width, rank), "down": ternary(rng, width, ffn, rank),
            "norm1": 1 + 0.1 * torch.randn(width, generator=gen, device="cuda"), "norm2": 1 + 0.1 * torch.randn(width, generator=gen, device="cuda")}


def random_adapter(out: int, inner: int, rank: int, gen):
    """A triple for AdaptedLayer.set_adapter: a tenth of what the projection itself does."""
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    return draw(rank, inner) / inner ** 0.5, draw(out, rank) / rank ** 0.5, 0.1


def pages(lengths, page_tokens: int):
    """A page table for sequences that will grow to `lengths`, and the number of pages it takes."""
    per = max(-(-n // page_tokens) for n in lengths)
    return torch.arange(len(lengths) * per, dtype=torch.int32, device="cuda").view(len(lengths), per), len(lengths) * per


def main() -> None:
    p = argparse.ArgumentParser()
    for name, value in (("width", 4096), ("heads", 32), ("kv-heads", 32), ("ffn", 16384), ("rank", 4096), ("sequences", 8), ("prompt", 512),
                        ("tokens", 32), ("adapters", 0), ("adapter-rank", 16), ("window", 0), ("sinks", 0)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    new = [max(1, a.prompt * (s + 1) // a.sequences) for s in range(a.sequences)]
    table, n_pages = pages([n + a.tokens for n in new], 64)
    weights = random_weights(a.width, a.heads, a.kv_heads, a.ffn, a.rank)
    if a.adapters:
        layer = AdaptedLayer(weights, a.heads, a.kv_heads, n_pages, n_adapters=a.adapters, adapter_rank=a.adapter_rank,
                             positions=max(new) + a.tokens, window=a.window, sinks=a.sinks)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(1)
        for i in range(a.adapters):
            layer.set_adapter(i, random_adapter(weights["qkv"].shape[0], a.width, a.adapter_rank, gen),
                              random_adapter(a.width, a.width, a.adapter_rank, gen))
        asked = torch.tensor([s % (a.adapters + 1) - 1 for s in range(a.sequences)], dtype=torch.int32, device="cuda")
    else:
        layer = ServedLayer(weights, a.heads, a.kv_heads, n_pages)
    layer.reserve(sum(new))
    start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    seq_len = torch.tensor(new, dtype=torch.int32, device="cuda")
    x = torch.randn(sum(new), a.width, device="cuda").to(torch.bfloat16)

    def timed(f):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        y = f()
        end.record()
        torch.cuda.synchronize()
        return y, begin.elapsed_time(end)

    def run(x, *batch):
        return layer.forward(x, torch.zeros_like(x), asked, *batch)[0] if a.adapters else layer.forward(x, *batch)

    run(x, table, seq_len, start, max(new))                  # (the same positions again below)
    y, ms = timed(lambda: run(x, table, seq_len, start, max(new)))
    print(f"prompts of {new} tokens: {ms:.3f} ms")
    token = y[start[1:].long() - 1]                          # the last row of each sequence
    times = []
    for _ in range(a.tokens):
        seq_len += 1
        token, ms = timed(lambda: run(token, table, seq_len))
        times.append(ms)
    print(f"{a.tokens} tokens for each of {a.sequences} sequences: {sorted(times)[len(times) // 2] * 1e3:.1f} us a token (median)")
    if layer.status():
        raise SystemExit(f"device status {layer.status()}")


if __name__ == "__main__":
    main()
