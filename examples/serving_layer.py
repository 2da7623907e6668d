"""A decoder layer as it is served: ternary feed-forward layers (TSVDLinear), dense projections in 8 bits (Int8Linear) and
attention over a key/value cache in 4 bits (KV4Cache).  Random weights; sizes of one OPT-6.7B layer unless told otherwise.

    python examples/serving_layer.py [--width 4096 --heads 32 --ffn 16384 --rank 4096 --sequences 8 --prompt 512 --tokens 32]

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

from paper_2308_07641_b200 import Int8Linear, KV4Cache, TSVDLinear, quantize  # noqa: E402


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
            "up": ternary(rng, ffn, width, rank), "down": ternary(rng, width, ffn, rank)}


def pages(lengths, page_tokens: int):
    """A page table for sequences that will grow to `lengths`, and the number of pages it takes."""
    per = max(-(-n // page_tokens) for n in lengths)
    return torch.arange(len(lengths) * per, dtype=torch.int32, device="cuda").view(len(lengths), per), len(lengths) * per


def main() -> None:
    p = argparse.ArgumentParser()
    for name, value in (("width", 4096), ("heads", 32), ("kv-heads", 32), ("ffn", 16384), ("rank", 4096), ("sequences", 8), ("prompt", 512),
                        ("tokens", 32)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    new = [max(1, a.prompt * (s + 1) // a.sequences) for s in range(a.sequences)]
    table, n_pages = pages([n + a.tokens for n in new], 64)
    layer = ServedLayer(random_weights(a.width, a.heads, a.kv_heads, a.ffn, a.rank), a.heads, a.kv_heads, n_pages)
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

    layer.forward(x, table, seq_len, start, max(new))        # (the same positions again below)
    y, ms = timed(lambda: layer.forward(x, table, seq_len, start, max(new)))
    print(f"prompts of {new} tokens: {ms:.3f} ms")
    token = y[start[1:].long() - 1]                          # the last row of each sequence
    times = []
    for _ in range(a.tokens):
        seq_len += 1
        token, ms = timed(lambda: layer.forward(token, table, seq_len))
        times.append(ms)
    print(f"{a.tokens} tokens for each of {a.sequences} sequences: {sorted(times)[len(times) // 2] * 1e3:.1f} us a token (median)")
    if layer.status():
        raise SystemExit(f"device status {layer.status()}")


if __name__ == "__main__":
    main()
