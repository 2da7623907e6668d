"""The serving operators against plain implementations in 64 bits.

Tolerances, from the arithmetic that include/tsvd_serving.h states (u16 = 2^-11 and u8 = 2^-8 are the unit roundoffs of
fp16 and bf16, u = 2^-24 that of fp32):
  8-bit rows, cache contents   equal: the definition is in fp32 and elementwise
  8-bit layer                  sum exact; product with two scales and the addition of the bias round at most 4 times:
                               4u (|sum scale wscale| + |bias|), and u8 |y| where y is bf16
  attention, bf16              scores: k as fp16 moves scale q.k by at most d = u16 scale sum |q k|, a softmax by at most
                               2d relative; p as fp16 (numerator and sum alike) 2 u16, v as fp16 u16, fp32 sums over n
                               positions below n u: (2 d + 3 u16 + 2 n u) sum p |v|, and u8 |out| for the result's rounding
  attention, fp32              the same with u in the place of u16, and 128-term dot products: d = 130 u scale sum |q k|;
                               exp within 4u
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U, U16, U8 = 2.0 ** -24, 2.0 ** -11, 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2308_07641_b200 import build
    build.build()


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


# ---- 8-bit rows ------------------------------------------------------------------------------------------------------


def _plain_quantize(x):
    """The definition, elementwise in fp32 on the host."""
    x = x.float().cpu().numpy()
    a = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(x.shape[0], np.float32)
    inv = np.zeros_like(a)
    np.divide(np.float32(1), a, out=inv, where=a >= np.float32(2.0 ** -100))
    inv = inv * np.float32(127)
    return np.rint(x * inv[:, None]).astype(np.int8), a * (np.float32(1) / np.float32(127))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 64, 0, 0), (5, 100, 12, 0), (2, 129, 7, 1), (4, 1001, 0, 3),
                                                 (3, 4096, 0, 0), (2, 4097, 0, 0), (1, 16384, 0, 0), (2, 20000, 8, 0), (1, 70001, 0, 0),
                                                 (700, 256, 0, 0), (2049, 33, 0, 0)])
def test_quantize_and_back(dtype, rows, cols, pad, shift):
    import torch
    from paper_2308_07641_b200 import dequantize, quantize
    g = _gen(rows * 1000 + cols)
    store = torch.randn(rows * (cols + pad) + shift, generator=g, device="cuda").mul_(3).to(_dtype(dtype))
    x = store[shift:].view(rows, cols + pad)[:, :cols]
    if rows > 2:
        x[1] = 0
        x[2] *= 1e-3
    q, scale = quantize(x)
    want_q, want_s = _plain_quantize(x)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(scale.cpu().numpy(), want_s)
    y = dequantize(q, scale)
    assert np.array_equal(y.cpu().numpy(), want_q.astype(np.float32) * want_s[:, None])
    yb = dequantize(q, scale, torch.bfloat16)
    assert torch.equal(yb, y.bfloat16())
    # q with rows that are not 16-byte aligned
    yo = dequantize(q.contiguous(), scale)
    assert torch.equal(yo, y)


def test_quantize_extreme_rows():
    import torch
    from paper_2308_07641_b200 import dequantize, quantize
    x = torch.zeros(7, 300, device="cuda")
    x[0, 5] = 1e-38           # too small for 127 / a: zeros
    x[1, :] = 3e38            # the largest magnitudes
    x[2, 7] = -2.0            # one value
    x[3, 299] = float("inf")
    x[4, 0] = float("nan")
    x[5, :] = torch.linspace(-1, 1, 300, device="cuda")
    q, scale = quantize(x)
    assert (q[0] == 0).all() and (q[6] == 0).all() and scale[6] == 0
    assert (q[1] == 127).all() and torch.isfinite(scale[1])
    assert q[2, 7] == -127 and q[2].count_nonzero() == 1
    assert not torch.isfinite(scale[3]) and not torch.isfinite(scale[4])       # visible in whatever uses it
    y = dequantize(q, scale)
    assert torch.isfinite(y[[0, 1, 2, 5, 6]]).all() and not torch.isfinite(y[[3, 4]]).any()
    assert q[5].abs().max() == 127 and (q[5].float().diff() >= 0).all()


def test_no_rows():
    import torch
    from paper_2308_07641_b200 import Int8Linear, KV4Cache, dequantize, quantize
    q, scale = quantize(torch.empty(0, 64, device="cuda"))
    assert q.shape == (0, 64) and dequantize(q, scale).shape == (0, 64)
    layer = Int8Linear(torch.ones(8, 64, dtype=torch.int8), torch.ones(8))
    assert layer(torch.empty(0, 64, device="cuda")).shape == (0, 8)
    cache = KV4Cache(2, 64, 4, 16)
    table, zero = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    e = torch.empty(0, 2, 64, device="cuda")
    cache.append(e, e, table, zero, start)
    assert cache.attend(e, table, zero, start).shape == (0, 2, 64)
    assert cache.read(0, table, zero, start)[0].shape == (0, 2, 64)
    torch.cuda.synchronize()
    assert cache.status() == 0


# ---- the 8-bit layer -------------------------------------------------------------------------------------------------


def _check_layer(y, x8, xs, w8, ws, bias):
    import torch
    total = x8.double().cpu() @ w8.double().cpu().T            # exact: below 2^53
    main = total * xs.double().cpu()[:, None] * ws.double().cpu()[None, :]
    b = torch.zeros(w8.shape[0], dtype=torch.float64) if bias is None else bias.double().cpu()
    want = main + b
    tol = 4 * U * (main.abs() + b.abs())
    if y.dtype == torch.bfloat16:
        tol = tol + U8 * want.abs()
    err = (y.double().cpu() - want).abs()
    assert (err <= tol + 1e-300).all(), f"worst {(err / (tol + 1e-300)).max():.3g} of the tolerance"


SIZES = [(1, 1, 1), (1, 128, 128), (2, 130, 127), (3, 64, 1000), (7, 1001, 300), (8, 4096, 512), (9, 256, 129), (16, 2048, 640),
         (17, 333, 257), (31, 128, 128), (33, 1000, 130), (64, 512, 512), (65, 640, 384), (100, 4096, 256), (128, 257, 1024),
         (129, 768, 770), (255, 384, 128), (257, 1001, 200), (300, 128, 2048), (513, 520, 640), (1025, 768, 384)]


@pytest.mark.parametrize("B,N,M", SIZES)
@pytest.mark.parametrize("dtype", ["i8", "bf16", "f32"])
def test_layer(B, N, M, dtype):
    import torch
    from paper_2308_07641_b200 import Int8Linear, quantize
    g = _gen(B * 7 + N * 3 + M)
    w8 = torch.randint(-127, 128, (M, N), generator=g, device="cuda", dtype=torch.int8)
    ws = torch.rand(M, generator=g, device="cuda") * 0.01 + 1e-4
    bias = torch.randn(M, generator=g, device="cuda") if (B + M) % 2 else None
    layer = Int8Linear(w8, ws, bias)
    if dtype == "i8":
        x8 = torch.randint(-128, 128, (B, N), generator=g, device="cuda", dtype=torch.int8)
        xs = torch.rand(B, generator=g, device="cuda") + 0.5
        _check_layer(layer(x8, xs), x8, xs, w8, ws, bias)
        from paper_2308_07641_b200 import binding
        _check_layer(layer(x8, xs, flags=binding.TSVD_FLAG_OUT_BF16), x8, xs, w8, ws, bias)
    else:
        x = (torch.randn(B, N, generator=g, device="cuda") * 2).to(_dtype(dtype))
        x8, xs = quantize(x)
        _check_layer(layer(x), x8, xs, w8, ws, bias)
    assert layer.status() == 0


def test_layer_strides_alignment_and_output_bounds():
    """Rows that are slices of wider ones, at odd addresses; nothing outside y's own rows and columns is written."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, binding, quantize
    g = _gen(5)
    for B, N, M in ((5, 200, 190), (70, 1000, 130), (300, 129, 333)):
        w8 = torch.randint(-127, 128, (M, N + 5), generator=g, device="cuda", dtype=torch.int8)[:, 3:3 + N]
        ws = torch.rand(M, generator=g, device="cuda")
        layer = Int8Linear(w8, ws)
        wide = torch.randint(-127, 128, (B * (N + 9) + 1,), generator=g, device="cuda", dtype=torch.int8)
        x8 = wide[1:].view(B, N + 9)[:, 2:2 + N]
        xs = torch.ones(B, device="cuda")
        frame = torch.full((B + 2, M + 6), 7.0, device="cuda")
        y = frame[1:B + 1, 3:3 + M]
        layer(x8, xs, out=y)
        _check_layer(y, x8, xs, w8, ws, None)
        frame[1:B + 1, 3:3 + M] = 7.0
        assert (frame == 7.0).all()
        xb = torch.randn(B, N + 3, generator=g, device="cuda").bfloat16()[:, 1:1 + N]
        frame16 = torch.full((B + 2, M + 6), 7.0, device="cuda", dtype=torch.bfloat16)
        layer(xb, out=frame16[1:B + 1, 3:3 + M])
        q, s = quantize(xb)
        _check_layer(frame16[1:B + 1, 3:3 + M], q, s, w8, ws, None)
        frame16[1:B + 1, 3:3 + M] = 7.0
        assert (frame16 == 7.0).all()
        with pytest.raises(binding.TSVDError):
            layer(x8[:, :-1])


def test_layer_extreme_sums():
    """The longest contraction with every product at its largest: the 32-bit sums do not wrap."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, binding
    N = binding.TSVD_I8_MAX_N
    w8 = torch.full((130, N), -128, dtype=torch.int8, device="cuda")
    w8[1] = 127
    layer = Int8Linear(w8, torch.ones(130, device="cuda"))
    for B in (1, 70):
        x8 = torch.full((B, N), -128, dtype=torch.int8, device="cuda")
        y = layer(x8)
        assert (y[:, 0].double() == np.float32(128.0 * 128 * N)).all() and (y[:, 1].double() == np.float32(-128.0 * 127 * N)).all()


def test_layer_reads_weights_from_the_host_and_keeps_its_own():
    import torch
    from paper_2308_07641_b200 import Int8Linear
    w8, ws, b = torch.randint(-127, 128, (70, 90), dtype=torch.int8), torch.rand(70), torch.randn(70)
    layer = Int8Linear(w8, ws, b)
    x8, xs = torch.randint(-127, 128, (4, 90), dtype=torch.int8, device="cuda"), torch.rand(4, device="cuda")
    keep = w8.clone()
    w8.zero_()
    _check_layer(layer(x8, xs), x8, xs, keep, ws, b)


@pytest.mark.parametrize("B", [1, 40, 300])
def test_layer_on_another_stream_and_in_a_graph(B):
    """Inputs change between replays; the results follow."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, quantize
    g = _gen(B)
    w = torch.randn(384, 512, generator=g, device="cuda")
    layer = Int8Linear(*quantize(w))
    layer.reserve(B, "bf16")
    x = torch.randn(B, 512, generator=g, device="cuda").bfloat16()
    y = torch.empty(B, 384, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, out=y)
    side.synchronize()
    want = layer(x)
    torch.cuda.synchronize()
    assert torch.equal(want, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(x, out=y)
    for k in range(3):
        x.copy_(torch.randn(B, 512, generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer(x), y)


def test_layer_zero_and_poisoned_tokens():
    import torch
    from paper_2308_07641_b200 import Int8Linear
    for B in (3, 70):
        layer = Int8Linear(torch.ones(130, 200, dtype=torch.int8), torch.ones(130), torch.full((130,), 0.5))
        x = torch.randn(B, 200, device="cuda")
        x[1] = 0
        x[2, 17] = float("nan")
        y = layer(x)
        assert (y[1] == 0.5).all() and not torch.isfinite(y[2]).any() and torch.isfinite(y[[0] + list(range(3, B))]).all()


# ---- the cache -------------------------------------------------------------------------------------------------------


def _plain_cached(x):
    """What the cache makes of [..., D] numbers, elementwise in fp32 on the host (the definition), as float64."""
    x = x.float().cpu().numpy()
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    most = np.float32(65000)
    lo, hi = np.clip(g.min(-1), -most, most), np.clip(g.max(-1), -most, most)
    step, base = ((hi - lo) * (np.float32(1) / np.float32(15))).astype(np.float16), lo.astype(np.float16)
    s = step.astype(np.float32)
    inv = np.zeros_like(s)
    np.divide(np.float32(1), s, out=inv, where=s > 0)
    code = np.clip(np.rint((g - base.astype(np.float32)[..., None]) * inv[..., None]), 0, 15)
    return (code.astype(np.float64) * step.astype(np.float64)[..., None] + base.astype(np.float64)[..., None]).reshape(x.shape)


class Batch:
    """Sequences with random keys and values, in a KV4Cache behind a shuffled page table and on the host as the plain
    implementation sees them."""

    def __init__(self, lens, Hkv, D, page, seed=0, dtype="bf16", spare_pages=3, offset=1.0):
        import torch
        from paper_2308_07641_b200 import KV4Cache
        g = _gen(seed + 17)
        self.lens, self.Hkv, self.D, self.page = list(lens), Hkv, D, page
        S, most = len(lens), max(max(lens), 1)
        per = -(-most // page) + 1
        n_pages = S * per + spare_pages
        self.cache = KV4Cache(Hkv, D, n_pages, page)
        self.table = torch.randperm(n_pages, generator=g, device="cuda")[:S * per].to(torch.int32).view(S, per).contiguous()
        self.seq_len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        rows = per * page
        # every page is filled to its end, with wild numbers behind the sequence: recycled pages
        k = torch.randn(S, rows, Hkv, D, generator=g, device="cuda") + offset * torch.randn(1, 1, Hkv, D, generator=g, device="cuda")
        v = torch.randn(S, rows, Hkv, D, generator=g, device="cuda")
        for s, n in enumerate(lens):
            k[s, n:] = 60000.0 * torch.sign(torch.randn(rows - n, Hkv, D, generator=g, device="cuda"))
            v[s, n:] = float("inf") * torch.sign(torch.randn(rows - n, Hkv, D, generator=g, device="cuda"))
            if n < rows:
                k[s, n, :, 0] = float("nan")
                v[s, n, :, 1] = float("nan")
        k, v = k.to(_dtype(dtype)), v.to(_dtype(dtype))
        full = torch.full((S,), rows, dtype=torch.int32, device="cuda")
        start = torch.arange(S + 1, dtype=torch.int32, device="cuda") * rows
        self.cache.append(k.view(-1, Hkv, D), v.view(-1, Hkv, D), self.table, full, start)
        self.k = [_plain_cached(k[s, :n]) for s, n in enumerate(lens)]
        self.v = [_plain_cached(v[s, :n]) for s, n in enumerate(lens)]

    def plain(self, q, new, causal, window, scale):
        """(out, sum p |v|, largest scale sum |q k| of a seen position) in 64 bits."""
        outs, sizes, reach = [], [], []
        q, first = q.double().cpu().numpy(), 0
        for s, n in enumerate(new):
            L = self.lens[s]
            qs = q[first:first + n]
            first += n
            G = q.shape[1] // self.Hkv
            k, v = np.repeat(self.k[s], G, axis=1), np.repeat(self.v[s], G, axis=1)
            score = np.einsum("ihd,jhd->ihj", qs, k) * scale
            size = np.einsum("ihd,jhd->ihj", np.abs(qs), np.abs(k)) * abs(scale)
            pos, j = np.arange(L - n, L)[:, None], np.arange(L)[None, :]
            see = (j <= pos) if causal else np.ones((n, L), bool)
            if window:
                see = see & (j > pos - window)
            score = np.where(see[:, None, :], score, -np.inf)
            top = score.max(-1, keepdims=True, initial=-np.inf)
            e = np.exp(score - np.where(np.isfinite(top), top, 0))
            total = e.sum(-1, keepdims=True)
            p = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
            outs.append(np.einsum("ihj,jhd->ihd", p, v))
            sizes.append(np.einsum("ihj,jhd->ihd", p, np.abs(v)))
            reach.append(np.where(see[:, None, :], size, 0).max(-1, initial=0.0))
        return np.concatenate(outs), np.concatenate(sizes), np.concatenate(reach)

    def check(self, H, new, causal=True, window=0, scale=None, dtype="bf16", seed=3, qmul=1.0, **kw):
        import torch
        n_rows = sum(new)
        q = (torch.randn(n_rows, H, self.D, generator=_gen(seed), device="cuda") * qmul).to(_dtype(dtype))
        start = None
        if any(n != 1 for n in new):
            start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        out = self.cache.attend(q, self.table, self.seq_len, start, causal=causal, window=window, scale=scale, **kw)
        sc = scale if scale is not None else 1 / math.sqrt(self.D)
        want, size, reach = self.plain(q, new, causal, window, sc)
        n = max(self.lens)
        u = U16 if dtype == "bf16" else U
        d = (1 if dtype == "bf16" else 130) * u * reach[..., None]
        tol = (2 * d + (3 if dtype == "bf16" else 12) * u + 2 * n * U) * size + (U8 if dtype == "bf16" else U) * np.abs(want) + 1e-30
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        err = np.abs(got - want) / tol
        assert err.max() <= 1, f"worst {err.max():.3g} of the tolerance at {np.unravel_index(err.argmax(), err.shape)}"
        assert (got[size.sum(-1) == 0] == 0).all()              # a row that sees nothing
        assert self.cache.status() == 0
        return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hkv,D,page,lens,new", [(1, 64, 16, [1], [1]), (3, 128, 16, [5, 17, 33], [1, 1, 1]), (2, 64, 48, [100, 3], [37, 3]),
                                                 (32, 128, 64, [70, 64, 65], [70, 1, 0]), (5, 64, 32, [0, 31, 64], [0, 31, 2])])
def test_append_and_read(dtype, Hkv, D, page, lens, new):
    import torch
    b = Batch(lens, Hkv, D, page, dtype=dtype)
    g = _gen(9)
    n = sum(new)
    # slices of one wide row, as a fused projection leaves them
    wide = (torch.randn(n, 3 * Hkv * D + 3, generator=g, device="cuda") * 5).to(_dtype(dtype))
    for off in (0, 3):
        k = wide[:, off + Hkv * D:off + 2 * Hkv * D].unflatten(1, (Hkv, D))
        v = wide[:, off + 2 * Hkv * D:off + 3 * Hkv * D].unflatten(1, (Hkv, D))
        start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        b.cache.append(k, v, b.table, b.seq_len, start)
        rk, rv = b.cache.read(n, b.table, b.seq_len, start)
        assert np.array_equal(rk.double().cpu().numpy(), _plain_cached(k)) and np.array_equal(rv.double().cpu().numpy(), _plain_cached(v))
        bk, bv = b.cache.read(n, b.table, b.seq_len, start, torch.bfloat16)
        assert torch.equal(bk, rk.bfloat16()) and torch.equal(bv, rv.bfloat16())
    # what lay before is untouched
    old = [L - m for L, m in zip(lens, new)]
    at = torch.tensor([0] + list(np.cumsum(old)), dtype=torch.int32, device="cuda")
    ok, ov = b.cache.read(sum(old), b.table, torch.tensor(old, dtype=torch.int32, device="cuda"), at)
    for s, m in enumerate(old):
        lo = int(sum(old[:s]))
        assert np.array_equal(ok[lo:lo + m].double().cpu().numpy(), b.k[s][:m])
        assert np.array_equal(ov[lo:lo + m].double().cpu().numpy(), b.v[s][:m])
    assert b.cache.status() == 0


def test_append_extreme_numbers():
    """Equal numbers, huge ones, infinities and NaN: what is kept is finite."""
    import torch
    from paper_2308_07641_b200 import KV4Cache
    cache = KV4Cache(1, 64, 1, 16)
    x = torch.zeros(6, 1, 64, device="cuda")
    x[0] = 3.25
    x[1, 0, ::2], x[1, 0, 1::2] = 1e30, -1e30
    x[2, 0, 5], x[2, 0, 40] = float("inf"), float("-inf")
    x[3, 0, 7] = float("nan")
    x[4] = float("nan")
    x[5, 0] = torch.linspace(-1e-6, 1e-6, 64, device="cuda")
    table, n = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([6], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    cache.append(x, x, table, n, start)
    k, v = cache.read(6, table, n, start)
    assert torch.isfinite(k).all() and torch.equal(k, v) and k.abs().max() < 65504
    assert (k[0] == 3.25).all() and (k[1, 0, ::2] > 64000).all() and (k[1, 0, 1::2] < -64000).all()


DECODE = [
    # lens, query heads, kv heads, D, page
    ([1], 1, 1, 64, 16), ([2], 2, 2, 128, 16), ([15], 4, 4, 64, 16), ([16], 4, 1, 128, 16), ([17], 8, 2, 64, 16), ([0, 33, 1], 3, 3, 128, 16),
    ([31, 0, 64, 63], 8, 1, 64, 32), ([100, 257, 1, 0, 16], 12, 4, 128, 48), ([700], 5, 1, 128, 64), ([513, 1024], 24, 2, 64, 64),
    ([1025], 32, 2, 128, 16), ([2000, 77], 33, 1, 64, 256), ([4099], 12, 12, 64, 16), ([6001, 10], 8, 8, 128, 1024), ([300] * 40, 16, 4, 128, 32),
    ([20000], 8, 2, 128, 256),
]


@pytest.mark.parametrize("lens,H,Hkv,D,page", DECODE)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_one_token_each(lens, H, Hkv, D, page, dtype):
    b = Batch(lens, Hkv, D, page, seed=H)
    out = b.check(H, [1] * len(lens), dtype=dtype)
    import torch
    again = b.check(H, [1] * len(lens), dtype=dtype, max_kv=max(max(lens), 1))
    if max(lens) < 64:
        assert torch.equal(out, again)
    b.check(H, [1] * len(lens), dtype=dtype, window=37)
    b.check(H, [1] * len(lens), dtype=dtype, causal=False, scale=0.3)


ROWS = [
    # lens, new, query heads, kv heads, D, page
    ([2], [2], 1, 1, 64, 16), ([10], [3], 4, 4, 128, 16), ([40], [8], 8, 2, 64, 16), ([50, 9, 128], [5, 9, 1], 8, 8, 128, 64),
    ([64], [64], 2, 2, 64, 16), ([130], [130], 3, 3, 128, 16), ([127, 129, 300], [127, 129, 33], 4, 2, 64, 32),
    ([500, 0, 77], [300, 0, 77], 6, 2, 128, 48), ([1100], [257], 8, 1, 128, 64), ([900], [900], 2, 1, 64, 128), ([260, 1, 256], [256, 1, 1], 4, 4, 128, 256),
    ([33, 600], [33, 40], 5, 1, 64, 16), ([2048], [1024], 2, 2, 128, 64), ([1500, 1499], [129, 700], 12, 3, 64, 64),
    # few rows behind a long context: blocks share the positions
    ([4000], [40], 2, 2, 128, 64), ([3001, 700], [65, 1], 8, 1, 64, 32), ([5000, 90, 0, 1300], [130, 90, 0, 33], 4, 2, 128, 16),
    # many sequences of unlike lengths, some without a row or a position
    ([(37 * i) % 301 for i in range(16)], [min((37 * i) % 301, (53 * i) % 190) for i in range(16)], 4, 4, 64, 16),
    ([(61 * i) % 700 for i in range(10)], [min((61 * i) % 700, (89 * i) % 400) for i in range(10)], 16, 4, 128, 32),
]


@pytest.mark.parametrize("lens,new,H,Hkv,D,page", ROWS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_several_rows(lens, new, H, Hkv, D, page, dtype):
    b = Batch(lens, Hkv, D, page, seed=H + 1)
    b.check(H, new, dtype=dtype)
    b.check(H, new, dtype=dtype, max_q=max(new), max_kv=max(lens), window=100)
    b.check(H, new, dtype=dtype, max_q=max(new), causal=False, window=65)
    b.check(H, new, dtype=dtype, max_q=max(new), causal=False, scale=-0.2)


@pytest.mark.parametrize("new", [1, 20, 200])
def test_attend_sharp_and_flat_softmax(new):
    """Scores of the order of hundreds (one position takes everything) and all equal."""
    b = Batch([777], 2, 128, 64, seed=4)
    b.check(4, [new], qmul=40.0)
    b.check(4, [new], qmul=0.0)
    b.check(4, [new], scale=0.0, window=300)
    b.check(4, [new], qmul=1e-30)


@pytest.mark.parametrize("new", [1, 200])
def test_attend_simple_path_agrees(new):
    import torch
    from paper_2308_07641_b200 import binding
    b = Batch([611], 2, 64, 32, seed=5)
    b.check(8, [new])
    b.check(8, [new], flags=binding.TSVD_FLAG_PATH_SIMPLE)
    torch.cuda.synchronize()


@pytest.mark.parametrize("lens,new", [([4000, 77], [1, 1]), ([500, 300], [200, 3])])
def test_attend_is_deterministic(lens, new):
    import torch
    b = Batch(lens, 4, 128, 64)
    first = b.check(8, new)
    for _ in range(4):
        assert torch.equal(first, b.check(8, new))


@pytest.mark.parametrize("new", [1, 9, 150])
def test_attend_strided_rows_and_output_bounds(new):
    """q as a slice of a fused projection, out inside a larger tensor; nothing else is written."""
    import torch
    H, Hkv, D = 8, 4, 64
    b = Batch([333, 200], Hkv, D, 32)
    n = 2 * new
    wide = torch.randn(n, H * D + 2 * Hkv * D, generator=_gen(1), device="cuda").bfloat16()
    q = wide[:, :H * D].unflatten(1, (H, D))
    frame = torch.full((n + 2, H * D + 16), 3.0, device="cuda", dtype=torch.bfloat16)
    out = frame[1:n + 1, 8:8 + H * D].unflatten(1, (H, D))
    start = torch.tensor([0, new, 2 * new], dtype=torch.int32, device="cuda")
    b.cache.attend(q, b.table, b.seq_len, start, max_q=new, out=out)
    want = b.cache.attend(q.contiguous(), b.table, b.seq_len, start, max_q=new)
    assert torch.equal(out, want)
    frame[1:n + 1, 8:8 + H * D] = 3.0
    assert (frame == 3.0).all()


def test_attend_refuses():
    import torch
    from paper_2308_07641_b200 import binding
    b = Batch([50], 2, 64, 16)
    q = torch.zeros(1, 4, 64, device="cuda", dtype=torch.bfloat16)
    def status(**kw):
        a = dict(q=q, page_table=b.table, seq_len=b.seq_len)
        a.update(kw)
        with pytest.raises(binding.TSVDError) as e:
            b.cache.attend(**a)
        return e.value.status
    assert status(q=torch.zeros(1, 3, 64, device="cuda", dtype=torch.bfloat16)) == binding.TSVD_E_SHAPE     # 3 heads over 2
    assert status(q=torch.zeros(1, 4, 32, device="cuda", dtype=torch.bfloat16)) == binding.TSVD_E_SHAPE
    assert status(q=q.half()) == binding.TSVD_E_DTYPE
    assert status(q=torch.zeros(2, 4, 64, device="cuda", dtype=torch.bfloat16)) == binding.TSVD_E_SHAPE     # 2 rows, 1 sequence
    assert status(seq_len=b.seq_len.long()) == binding.TSVD_E_DTYPE
    assert status(page_table=b.table[0]) == binding.TSVD_E_SHAPE
    assert status(window=-1) == binding.TSVD_E_SHAPE
    assert status(scale=float("nan")) == binding.TSVD_E_SHAPE
    assert status(flags=binding.TSVD_FLAG_PATH_TENSOR) == binding.TSVD_E_DTYPE
    odd = torch.zeros(4 * 64 + 1, device="cuda", dtype=torch.bfloat16)[1:].view(1, 4, 64)
    assert status(q=odd) == binding.TSVD_E_ALIGN
    assert b.cache.status() == 0


@pytest.mark.parametrize("new", [1, 6, 140])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_and_lengths_out_of_range(new, dtype):
    """A page number outside the pool and a length beyond the pages: those positions are not seen, the status says so,
    and nothing else changes."""
    import torch
    from paper_2308_07641_b200 import KV4Cache, binding
    D, page = 64, 16
    g = _gen(2)
    L = 160
    x = torch.randn(L, 1, D, generator=g, device="cuda").to(_dtype(dtype))
    start, n = torch.tensor([0, L], dtype=torch.int32, device="cuda"), torch.tensor([L], dtype=torch.int32, device="cuda")
    cache = KV4Cache(1, D, 10, page)
    table = torch.arange(10, dtype=torch.int32, device="cuda").view(1, 10)
    cache.append(x, x, table, n, start)
    assert cache.status() == 0
    q = torch.randn(new, 1, D, generator=g, device="cuda").to(_dtype(dtype))
    qs = torch.tensor([0, new], dtype=torch.int32, device="cuda")
    for bad in (-1, 10, 1 << 30):
        broken = table.clone()
        broken[0, 3] = bad
        out = cache.attend(q, broken, n, qs, max_q=new, causal=False)
        torch.cuda.synchronize()
        assert cache.status() == binding.TSVD_E_INDEX and cache.status() == 0
        # the same as without those 16 positions
        other = KV4Cache(1, D, 9, page)
        keep = torch.cat((x[:48], x[64:]))
        short = torch.tensor([L - 16], dtype=torch.int32, device="cuda")
        t9 = torch.arange(9, dtype=torch.int32, device="cuda").view(1, 9)
        other.append(keep, keep, t9, short, torch.tensor([0, L - 16], dtype=torch.int32, device="cuda"))
        want = other.attend(q, t9, short, qs, max_q=new, causal=False)
        tol = 2 ** -6 if dtype == "bf16" else 2 ** -18
        assert (out.double() - want.double()).abs().max() <= tol * want.double().abs().max()
    # longer than its pages, in attend, append and read
    out = cache.attend(q, table[:, :5].contiguous(), n, qs, max_q=new, causal=False)
    assert torch.isfinite(out).all() and cache.status() == binding.TSVD_E_INDEX
    before = cache.read(L, table, n, start)[0]
    cache.append(x + 1, x + 1, table[:, :5].contiguous(), n, start)
    assert cache.status() == binding.TSVD_E_INDEX
    after = cache.read(L, table, n, start)[0]
    assert torch.equal(after[80:], before[80:]) and not torch.equal(after[:80], before[:80])
    k, _ = cache.read(L, table[:, :5].contiguous(), n, start)
    assert cache.status() == binding.TSVD_E_INDEX and (k[80:] == 0).all() and (k[:80] != 0).any()
    # more new rows than positions: the ones before position 0 see nothing under a causal mask
    few = torch.tensor([2], dtype=torch.int32, device="cuda")
    out = cache.attend(q, table, few, qs, max_q=new)
    assert (out[:max(0, new - 2)] == 0).all() and (out[max(0, new - 2):] != 0).any()
    assert cache.status() == 0


def test_pool_beyond_four_gigabytes():
    """Pages whose byte offsets pass 32 bits."""
    import torch
    from paper_2308_07641_b200 import KV4Cache
    Hkv, D, page = 32, 128, 64
    n_pages = (5 << 30) // (Hkv * page * D * 5 // 4)
    cache = KV4Cache(Hkv, D, n_pages, page)
    g = _gen(0)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    for L, new in ((150, 1), (150, 150)):
        x, y = (torch.randn(L, Hkv, D, generator=g, device="cuda").bfloat16() for _ in range(2))
        n, start = torch.tensor([L], dtype=torch.int32, device="cuda"), torch.tensor([0, L], dtype=torch.int32, device="cuda")
        cache.append(x, y, table, n, start)
        k, v = cache.read(L, table, n, start)
        assert np.array_equal(k.double().cpu().numpy(), _plain_cached(x)) and np.array_equal(v.double().cpu().numpy(), _plain_cached(y))
        q = torch.randn(new, Hkv, D, generator=g, device="cuda").bfloat16()
        out = cache.attend(q, table, n, torch.tensor([0, new], dtype=torch.int32, device="cuda"), max_q=new)
        small = KV4Cache(Hkv, D, 3, page)
        t3 = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)
        small.append(x, y, t3, n, start)
        want = small.attend(q, t3, n, torch.tensor([0, new], dtype=torch.int32, device="cuda"), max_q=new)
        assert torch.equal(out, want)
    assert cache.status() == 0


@pytest.mark.parametrize("new", [1, 64])
def test_lengths_change_under_a_graph(new):
    """seq_len, q_start and the page table are read on the device: a captured call follows them."""
    import torch
    b = Batch([900, 40, 333], 2, 64, 32)
    q = torch.randn(3 * new, 4, 64, generator=_gen(6), device="cuda").bfloat16()
    start = torch.arange(4, dtype=torch.int32, device="cuda") * new
    seq_len, table = b.seq_len.clone(), b.table.clone()
    out = torch.empty_like(q)
    b.cache.attend(q, table, seq_len, start, max_q=new, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.cache.attend(q, table, seq_len, start, max_q=new, out=out)
    for lens in ([900, 40, 333], [64, 70, 1000], [500, 64, 65]):
        lens = [min(n, b.table.shape[1] * b.page) for n in lens]
        seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        perm = torch.randperm(3, generator=torch.Generator().manual_seed(sum(lens)))
        table.copy_(b.table[perm.cuda()])
        graph.replay()
        torch.cuda.synchronize()
        want = b.cache.attend(q, table, seq_len, start, max_q=new)
        assert torch.equal(out, want)


def test_another_stream():
    import torch
    b = Batch([1200], 2, 128, 64)
    q = torch.randn(1, 8, 128, generator=_gen(8), device="cuda").bfloat16()
    want = b.cache.attend(q, b.table, b.seq_len)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = b.cache.attend(q, b.table, b.seq_len)
    side.synchronize()
    assert torch.equal(got, want)
