"""Append with the rotation by position, and attention with first positions that a window does not hide.

Rotation: products and sums are single fp32 operations in a stated order, so queries and the cache's contents are equal to the
plain form's, bit for bit.  The table: angles in 64 bits, of a position below 2^20 off by less than 2^-33, cosines and sines
rounded once: 2^-24 off at most, 2^-25 by the rounding.  Attention: tolerances as in test_serving_gpu.py.
"""
import math

import numpy as np
import pytest

from tests.test_serving_gpu import Batch, _dtype, _gen, _plain_cached

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2308_07641_b200 import build
    build.build()


# ---- rotation ------------------------------------------------------------------------------------------------------------


def _turn(x, pos, table, interleaved):
    """The definition in fp32 on the host: x [rows, heads, D], pos [rows]."""
    x, t = x.float().cpu().numpy().copy(), table.cpu().numpy()[pos]
    half = t.shape[1] // 2
    c, s = t[:, None, :half], t[:, None, half:]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    u, v = x[..., a].copy(), x[..., b].copy()
    x[..., a] = u * c - v * s
    x[..., b] = v * c + u * s
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,D,page,lens,new,turned,interleaved", [
    (1, 1, 64, 16, [1], [1], 64, False), (3, 3, 128, 16, [5, 17, 33], [1, 1, 1], 128, False), (4, 2, 64, 48, [100, 3], [37, 3], 32, True),
    (32, 32, 128, 64, [70, 64, 65], [70, 1, 0], 128, True), (5, 5, 64, 32, [0, 31, 64], [0, 31, 2], 24, False), (16, 2, 128, 16, [40], [9], 64, False),
    (8, 1, 64, 16, [33], [20], 2, False), (8, 8, 128, 32, [20, 90], [20, 5], 50, True), (6, 3, 128, 16, [700], [1], 96, False),
    (12, 12, 64, 64, [5000, 66000], [3, 4], 48, True), (0, 2, 64, 16, [20], [6], 64, False), (64, 8, 128, 16, [19], [19], 126, False)])
def test_append_rotated(dtype, H, Hkv, D, page, lens, new, turned, interleaved):
    import torch
    from paper_2308_07641_b200 import KV4Cache, rotary_table
    g = _gen(9)
    n, S, per = sum(new), len(lens), -(-max(lens) // page)
    pages = S * per
    cache = KV4Cache(Hkv, D, pages, page)
    lines = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(S, per)
    seq_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    table = rotary_table(max(lens), turned)
    pos = np.concatenate([np.arange(L - m, L) for L, m in zip(lens, new)])
    # slices of one wide row, as a fused projection leaves them; off 16-byte boundaries the second time
    wide = (torch.randn(n, (H + 2 * Hkv) * D + 8, generator=g, device="cuda") * 5).to(_dtype(dtype))
    for off in (0, 3):
        q, k, v = (wide[:, off + a * D:off + b * D].unflatten(1, (b - a, D)) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv))) \
            if H else (None, *(wide[:, off + a * D:off + (a + Hkv) * D].unflatten(1, (Hkv, D)) for a in (0, Hkv)))
        got = cache.append_rotated(q, k, v, table, lines, seq_len, start, interleaved=interleaved)
        if H:
            want = torch.from_numpy(_turn(q, pos, table, interleaved)).to(_dtype(dtype))
            assert got.dtype == q.dtype and torch.equal(got.cpu(), want)
        else:
            assert got is None
        rk, rv = cache.read(n, lines, seq_len, start)
        assert np.array_equal(rk.double().cpu().numpy(), _plain_cached(torch.from_numpy(_turn(k, pos, table, interleaved))))
        assert np.array_equal(rv.double().cpu().numpy(), _plain_cached(v))
    assert cache.status() == 0


def test_table():
    import torch
    from paper_2308_07641_b200 import rotary_table
    for positions, turned, base in ((1, 2, 10000.0), (77, 64, 10000.0), (200000, 128, 500000.0)):
        t = rotary_table(positions, turned, base)
        rate = base ** (-torch.arange(0, turned, 2, dtype=torch.float64, device="cuda") / turned)
        a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * rate
        assert t.shape == (positions, turned) and (t.double() - torch.cat((a.cos(), a.sin()), 1)).abs().max() <= 2.0 ** -24
    rates = torch.tensor([0.5, 0.001], dtype=torch.float64)
    t = rotary_table(9, 4, rates=rates, amplitude=1.25)
    a = torch.arange(9, dtype=torch.float64)[:, None] * rates
    assert (t.double().cpu() - 1.25 * torch.cat((a.cos(), a.sin()), 1)).abs().max() <= 1.25 * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rotated_rows_out_of_range(dtype):
    """Positions behind the table, before 0, outside the pages; rows of no sequence."""
    import torch
    from paper_2308_07641_b200 import KV4Cache, binding, rotary_table
    g = _gen(2)
    D, H = 64, 2
    cache = KV4Cache(H, D, 6, 16)
    table = rotary_table(20, D)
    lines = torch.tensor([[0, 1], [2, 99], [4, 5]], dtype=torch.int32, device="cuda")
    seq_len = torch.tensor([24, 18, 2], dtype=torch.int32, device="cuda")
    start = torch.tensor([1, 7, 10, 14], dtype=torch.int32, device="cuda")           # rows 0, 14 and 15: nobody's
    q, k, v = (torch.randn(16, H, D, generator=g, device="cuda").to(_dtype(dtype)) for _ in range(3))
    from paper_2308_07641_b200 import serving
    fill = lambda shape, strides, **kw: torch.full(shape, 7.0, **kw)  # noqa: E731
    empty, serving._empty = serving._empty, fill
    try:
        out = cache.append_rotated(q, k, v, table, lines, seq_len, start)
    finally:
        serving._empty = empty
    torch.cuda.synchronize()
    assert cache.status() == binding.TSVD_E_INDEX and cache.status() == 0
    assert (out[[0, 14, 15]] == 7).all()
    pos = [18, 19, 20, 21, 22, 23, 15, 16, 17, -2, -1, 0, 1]                         # of rows 1 .. 13
    known = [0 <= p < 20 for p in pos]
    want = _turn(q[1:14], np.array([p if ok else 0 for p, ok in zip(pos, known)]), table, False) * np.array(known)[:, None, None]
    assert torch.equal(out[1:14].cpu(), torch.from_numpy(want).to(_dtype(dtype)))
    rk, rv = cache.read(16, lines, seq_len, start)
    kept = [ok and not (6 <= i < 9 and p >= 16) for i, (p, ok) in enumerate(zip(pos, known))]       # (page 99)
    want = _plain_cached(torch.from_numpy(_turn(k[1:14], np.array([p if ok else 0 for p, ok in zip(pos, known)]), table, False)))
    assert np.array_equal(rk[1:14].double().cpu().numpy(), want * np.array(kept)[:, None, None])
    assert (rk[[0, 14, 15]] == 0).all() and (rv[[0, 14, 15]] == 0).all()


def test_rotated_is_append_of_turned_keys():
    """Behind each other in a chain with the attention, on a side stream, in a graph: what append of turned keys gives."""
    import torch
    from paper_2308_07641_b200 import KV4Cache, rotary_table
    g = _gen(6)
    D, H, Hkv, S = 128, 8, 2, 5
    caches = [KV4Cache(Hkv, D, S * 8, 16) for _ in range(2)]
    lines = torch.arange(S * 8, dtype=torch.int32, device="cuda").view(S, 8)
    table = rotary_table(128, D)
    seq_len = torch.zeros(S, dtype=torch.int32, device="cuda")
    q, k, v = (torch.empty(S, h, D, device="cuda") for h in (H, Hkv, Hkv))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        t = caches[0].append_rotated(q, k, v, table, lines, seq_len)
        return t, caches[0].attend(t, lines, seq_len)

    with torch.cuda.graph(graph, stream=side):
        turned, out = step()
    for i in range(20):
        for t in (q, k, v):
            t.normal_()
        seq_len.add_(1)
        graph.replay()
        pos = (seq_len - 1).cpu().numpy()
        tk, tq = (torch.from_numpy(_turn(t, pos, table, False)).cuda() for t in (k, q))
        caches[1].append(tk, v, lines, seq_len)
        assert torch.equal(turned, tq) and torch.equal(out, caches[1].attend(tq, lines, seq_len))
    assert caches[0].status() == 0


# ---- first positions beside a window --------------------------------------------------------------------------------------


class Sinks(Batch):
    """Batch with `sinks` first positions exempt from the window in the plain form."""

    def plain(self, q, new, causal, window, scale):
        outs, sizes, reach = [], [], []
        q, first = q.double().cpu().numpy(), 0
        for s, n in enumerate(new):
            L, G = self.lens[s], q.shape[1] // self.Hkv
            qs = q[first:first + n]
            first += n
            k, v = np.repeat(self.k[s], G, axis=1), np.repeat(self.v[s], G, axis=1)
            pos, j = np.arange(L - n, L)[:, None], np.arange(L)[None, :]
            see = (j <= pos) if causal else np.ones((n, L), bool)
            see = see & ((j > pos - window) | (j < self.sinks))
            score = np.where(see[:, None, :], np.einsum("ihd,jhd->ihj", qs, k) * scale, -np.inf)
            size = np.einsum("ihd,jhd->ihj", np.abs(qs), np.abs(k)) * abs(scale)
            top = score.max(-1, keepdims=True, initial=-np.inf)
            e = np.exp(score - np.where(np.isfinite(top), top, 0))
            total = e.sum(-1, keepdims=True)
            p = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
            outs.append(np.einsum("ihj,jhd->ihd", p, v))
            sizes.append(np.einsum("ihj,jhd->ihd", p, np.abs(v)))
            reach.append(np.where(see[:, None, :], size, 0).max(-1, initial=0.0))
        return np.concatenate(outs), np.concatenate(sizes), np.concatenate(reach)

    def check_sinks(self, H, new, window, sinks, **kw):
        self.sinks = sinks
        return self.check(H, new, window=window, sinks=sinks, **kw)


# (window, first positions): next to nothing, ends inside units and tiles, borders that touch, first positions beyond the window
WINDOWS = [(1, 1), (5, 4), (37, 3), (64, 32), (100, 33), (129, 128), (200, 131), (16, 300), (700, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,H,Hkv,D,page", [
    ([1], 1, 1, 64, 16), ([2], 2, 2, 128, 16), ([17], 8, 2, 64, 16), ([0, 33, 1], 3, 3, 128, 16), ([31, 0, 64, 63], 8, 1, 64, 32),
    ([100, 257, 1, 0, 16], 12, 4, 128, 48), ([513, 1024], 24, 2, 64, 64), ([1025], 32, 2, 128, 16), ([2000, 77], 33, 1, 64, 256),
    ([4099], 12, 12, 64, 16), ([300] * 40, 16, 4, 128, 32), ([6001, 10], 8, 8, 128, 1024)])
def test_sinks_one_token_each(lens, H, Hkv, D, page, dtype):
    b = Sinks(lens, Hkv, D, page, seed=H)
    for window, sinks in WINDOWS:
        b.check_sinks(H, [1] * len(lens), window, sinks, dtype=dtype)
    b.check_sinks(H, [1] * len(lens), 50, 20, dtype=dtype, causal=False, scale=-0.3)


@pytest.mark.parametrize("lens,new,H,Hkv,D,page", [
    ([10], [3], 4, 4, 128, 16), ([40], [8], 8, 2, 64, 16), ([50, 9, 128], [5, 9, 1], 8, 8, 128, 64), ([900, 30], [7, 2], 16, 2, 128, 16),
    ([64], [64], 2, 2, 64, 16), ([127, 129, 300], [127, 129, 33], 4, 2, 64, 32), ([500, 0, 77], [300, 0, 77], 6, 2, 128, 48),
    ([1100], [257], 8, 1, 128, 64), ([900], [900], 2, 1, 64, 128), ([33, 600], [33, 40], 5, 1, 64, 16), ([2048], [1024], 2, 2, 128, 64),
    ([1500, 1499], [129, 700], 12, 3, 64, 64), ([4000], [40], 2, 2, 128, 64), ([5000, 90, 0, 1300], [130, 90, 0, 33], 4, 2, 128, 16),
    ([(61 * i) % 700 for i in range(10)], [min((61 * i) % 700, (89 * i) % 400) for i in range(10)], 16, 4, 128, 32)])
def test_sinks_several_rows(lens, new, H, Hkv, D, page):
    b = Sinks(lens, Hkv, D, page, seed=H)
    for window, sinks in WINDOWS:
        b.check_sinks(H, new, window, sinks, max_q=max(new))
    b.check_sinks(H, new, 90, 40, causal=False, scale=0.2, max_q=max(new))
    b.check_sinks(H, new, 60, 70, dtype="f32", max_q=max(new))


@pytest.mark.parametrize("lens,new", [([700, 33], [1, 1]), ([700, 90], [200, 9]), ([6000], [64])])
def test_sinks_that_change_nothing(lens, new):
    """None of them, or no window: the bits of the call without; a window over everything: what no window gives, within tolerance."""
    import torch
    b = Sinks(lens, 2, 64, 32)
    q = torch.randn(sum(new), 4, 64, generator=_gen(3), device="cuda").bfloat16()
    start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
    call = lambda **kw: b.cache.attend(q, b.table, b.seq_len, start, max_q=max(new), **kw)  # noqa: E731
    assert torch.equal(call(window=50, sinks=0), call(window=50))
    assert torch.equal(call(window=0, sinks=9), call())
    b.check_sinks(4, new, 10000, 5, max_q=max(new))
    assert torch.equal(call(window=50, sinks=9), call(window=50, sinks=9))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 20, 100, 300])
@pytest.mark.parametrize("sinks,gone", [(20, (3, 43)), (4, (1, 31)), (16, (1, 43)), (160, (10, 37))])
def test_what_the_window_hides_is_not_read(new, sinks, gone, dtype):
    """Pages between the first positions and the window may be gone (their numbers out of range)."""
    b = Sinks([2000], 2, 64, 16)
    b.sinks = sinks
    window = 2000 - new + 1 - (16 * gone[1] + 5)             # the first row sees from position 16 gone[1] + 5 on
    b.table[0, gone[0]:gone[1]] = -7
    b.check(4, [new], window=window, sinks=sinks, max_q=new, dtype=dtype)


@pytest.mark.parametrize("lens,new,H,Hkv,D", [([500], [1], 2, 2, 64), ([9000, 70], [1, 1], 8, 2, 128), ([400, 300], [3, 3], 16, 4, 64),
                                              ([600], [300], 4, 2, 128), ([3000], [40], 4, 4, 64)])
def test_waits_give_up_with_sinks(lens, new, H, Hkv, D):
    import torch
    from tests.test_serving_calls_gpu import _stalled
    b = Batch(lens, Hkv, D, 64, seed=H)
    q = torch.randn(sum(new), H, D, generator=_gen(5), device="cuda").bfloat16()
    start = torch.tensor([0] + [sum(new[:i + 1]) for i in range(len(new))], dtype=torch.int32, device="cuda")
    _stalled(lambda flags: b.cache.attend(q, b.table, b.seq_len, start, max_q=max(new), flags=flags, window=200, sinks=70), b.cache.status)


def test_lengths_change_under_a_graph_with_sinks():
    import torch
    lens = [400, 90, 1000]
    b = Sinks(lens, 2, 128, 32)
    q = torch.randn(3, 8, 128, generator=_gen(1), device="cuda").bfloat16()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.cache.attend(q, b.table, b.seq_len, window=150, sinks=6)
    for n in (lens, [1, 89, 300], [0, 7, 160]):
        b.seq_len.copy_(torch.tensor(n))
        graph.replay()
        assert torch.equal(out, b.cache.attend(q, b.table, b.seq_len, window=150, sinks=6))
    assert b.cache.status() == 0 and math.isfinite(float(out.sum()))
