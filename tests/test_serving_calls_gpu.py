"""The serving operators where a call meets its surroundings: devices, streams, launches in a chain, rows of unlike size."""
import ctypes
import math

import numpy as np
import pytest

from tests.test_serving_gpu import U, U8, U16, Batch, _check_layer, _gen, _plain_cached

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2308_07641_b200 import build
    build.build()


def test_a_handle_of_another_device_is_refused():
    """A handle's first field is its device (struct tsvd_i8_s, tsvd_kv4_s).  Every call that would launch or allocate on the
    current device says TSVD_E_CUDA where that is another one."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, KV4Cache, binding
    layer = Int8Linear(torch.ones(8, 64, dtype=torch.int8), torch.ones(8))
    cache = KV4Cache(2, 64, 4, 16)
    x = torch.ones(1, 64, device="cuda")
    k = torch.ones(1, 2, 64, device="cuda")
    table, n = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    calls = [lambda: layer(x), lambda: layer.reserve(5000, "f32"), lambda: cache.append(k, k, table, n), lambda: cache.read(1, table, n),
             lambda: cache.attend(k, table, n)]
    at = [ctypes.c_int.from_address(h.handle) for h in (layer, cache)]
    here = torch.cuda.current_device()
    assert [d.value for d in at] == [here, here]
    launches = binding.tsvd_launch_count()
    for d in at:
        d.value = here + 1
    try:
        for call in calls:
            with pytest.raises(binding.TSVDError) as e:
                call()
            assert e.value.status == binding.TSVD_E_CUDA
        assert layer.status() == binding.TSVD_E_CUDA and cache.status() == binding.TSVD_E_CUDA
        assert binding.tsvd_launch_count() == launches
    finally:
        for d in at:
            d.value = here
    for call in calls:
        call()
    torch.cuda.synchronize()
    assert layer.status() == 0 and cache.status() == 0


def test_layers_on_two_streams():
    """Products whose contraction clusters share (few tokens, 18 row tiles, and smaller ones), side by side on two streams."""
    import torch
    from paper_2308_07641_b200 import Int8Linear
    sizes = [(2304, 4096, 1), (4096, 2048, 32), (640, 4096, 33), (1001, 770, 197)]
    layers, inputs = [], []
    for M, N, B in sizes:
        g = _gen(M + B)
        w8 = torch.randint(-127, 128, (M, N), generator=g, device="cuda", dtype=torch.int8)
        ws = torch.rand(M, generator=g, device="cuda") * 0.01 + 1e-4
        x8 = torch.randint(-127, 128, (B, N), generator=g, device="cuda", dtype=torch.int8)
        xs = torch.rand(B, generator=g, device="cuda") + 0.5
        pair = [Int8Linear(w8, ws) for _ in range(2)]
        for layer in pair:
            layer.reserve(B, "i8")
        layers.append(pair)
        inputs.append((x8, xs, w8, ws))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = {}
    for _ in range(10):
        for i, (x8, xs, _, _) in enumerate(inputs):
            for k, stream in enumerate(streams):
                with torch.cuda.stream(stream):
                    outs[i, k] = layers[(i + k) % len(sizes)][k](*inputs[(i + k) % len(sizes)][:2])
    torch.cuda.synchronize()
    for (i, k), y in outs.items():
        x8, xs, w8, ws = inputs[(i + k) % len(sizes)]
        _check_layer(y, x8, xs, w8, ws, None)
    assert all(layer.status() == 0 for pair in layers for layer in pair)


@pytest.mark.parametrize("D,new", [(64, 200), (128, 200), (64, 1)])
def test_append_attend_and_layer_in_a_chain(D, new):
    """Every kernel may start before the one ahead of it has ended; results are those of calls that wait for each other."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, quantize
    H = 2048 // D
    b = Batch([new + 300, new + 77, new], H, D, 64, seed=D)
    rows = 3 * new
    g = _gen(D)
    layer = Int8Linear(*quantize(torch.randn(4096, 2048, generator=g, device="cuda")))
    layer.reserve(32, "bf16")
    q, k, v = (torch.randn(rows, H, D, generator=g, device="cuda").bfloat16() for _ in range(3))
    start = torch.arange(4, dtype=torch.int32, device="cuda") * new

    def chain(wait):
        b.cache.append(k, v, b.table, b.seq_len, start)
        wait()
        a = b.cache.attend(q, b.table, b.seq_len, start, max_q=new)
        wait()
        return layer(a.view(rows, 2048)[:32])

    want = chain(torch.cuda.synchronize)
    torch.cuda.synchronize()
    outs = [chain(lambda: None) for _ in range(20)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in outs)
    assert layer.status() == 0 and b.cache.status() == 0


@pytest.mark.parametrize("lens,new,H,Hkv,D", [([300, 77], [150, 40], 4, 4, 128), ([500, 90], [70, 70], 16, 4, 64), ([2500], [40], 8, 8, 128),
                                              ([300, 50], [1, 1], 16, 2, 128)])
def test_rows_of_unlike_size(lens, new, H, Hkv, D):
    """A row's result does not depend on the rows beside it, whichever kernel takes them: neighbours 2^18 to 2^30 times larger,
    infinite or NaN leave it within the tolerance of its own arithmetic (that of test_serving_gpu), and the kernel for many rows
    changes no bit of it.  (Tokens and heads alike are rows.)"""
    import torch
    b = Batch(lens, Hkv, D, 64, seed=D + H)
    n = sum(new)
    g = _gen(n)
    sizes = torch.tensor([1.0, 2.0 ** -18, 2.0 ** -22, 2.0 ** -26, 2.0 ** -30], device="cuda")
    mul = sizes[torch.randint(0, 5, (n, H, 1), generator=g, device="cuda")] * 2.0 ** 18
    b.check(H, new, qmul=mul, max_q=max(new))
    b.check(H, new, qmul=mul, max_q=max(new), scale=-0.1, causal=False)
    q = torch.randn(n, H, D, generator=g, device="cuda").bfloat16()
    start = torch.tensor([0] + [sum(new[:i + 1]) for i in range(len(new))], dtype=torch.int32, device="cuda")
    kw = dict(max_q=max(new), max_kv=max(lens))
    alone = b.cache.attend(q, b.table, b.seq_len, start, **kw)
    want, size, reach = b.plain(q, new, True, 0, 1 / math.sqrt(D))
    tol = (2 * U16 * reach[..., None] + 3 * U16 + 2 * max(lens) * U) * size + U8 * np.abs(want)
    own = torch.rand(n, H, generator=g, device="cuda") < 0.5
    at = own.cpu().numpy()
    for bad in (2.0 ** 18, 2.0 ** 30, 1e38, float("inf"), float("nan")):
        every, one = torch.where(own[..., None], q, q * bad), q.clone()
        one[..., 3] = torch.where(own, q[..., 3], bad)       # one number of a row is enough
        for other in (every, one):
            got = b.cache.attend(other, b.table, b.seq_len, start, **kw)
            assert (np.abs(got.double().cpu().numpy() - want)[at] <= tol[at]).all(), bad
            if max(new) * (H // Hkv) > 16:
                assert torch.equal(got[own], alone[own]), bad
    torch.cuda.synchronize()
    assert b.cache.status() == 0


def test_a_new_cache_on_another_stream():
    """A pool is zeroed before its creation returns: what a stream that waits for nothing puts into it at once stays there.  (6 GB,
    a millisecond of zeros; the appended positions lie at its end.)"""
    import torch
    from paper_2308_07641_b200 import KV4Cache
    Hkv, D, page = 32, 128, 64
    n_pages = (6 << 30) // (Hkv * page * D * 5 // 4)
    side = torch.cuda.Stream()
    x = torch.randn(100, Hkv, D, generator=_gen(3), device="cuda").bfloat16()
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    n, start = torch.tensor([100], dtype=torch.int32, device="cuda"), torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    want = _plain_cached(x)
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            cache = KV4Cache(Hkv, D, n_pages, page)
            cache.append(x, x, table, n, start)
        torch.cuda.synchronize()
        k, v = cache.read(100, table, n, start)
        assert np.array_equal(k.double().cpu().numpy(), want) and np.array_equal(v.double().cpu().numpy(), want)
        cache.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_sequence(dtype):
    """q_start may be a piece of a longer one: rows before its first number and behind its last are nobody's."""
    import torch
    Hkv, D = 2, 64
    b = Batch([90, 200], Hkv, D, 16, seed=7, dtype=dtype)
    kind = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    for new in (1, 30):
        n = 2 * new + 10
        start = torch.tensor([6, 6 + new, 6 + 2 * new], dtype=torch.int32, device="cuda")
        mine = slice(6, 6 + 2 * new)
        whole = torch.tensor([0, 90, 290], dtype=torch.int32, device="cuda")
        before = b.cache.read(290, b.table, b.seq_len, whole)
        k, v = (torch.randn(n, Hkv, D, generator=_gen(new + i), device="cuda").to(kind) for i in range(2))
        b.cache.append(k, v, b.table, b.seq_len, start)
        after = b.cache.read(290, b.table, b.seq_len, whole)
        new_at = torch.zeros(290, dtype=torch.bool, device="cuda")
        new_at[90 - new:90] = True
        new_at[290 - new:] = True
        for old, now, x in zip(before, after, (k, v)):
            assert torch.equal(old[~new_at], now[~new_at])
            assert np.array_equal(now[new_at].double().cpu().numpy(), _plain_cached(x[mine]))
        for got, now in zip(b.cache.read(n, b.table, b.seq_len, start), after):
            assert torch.equal(got[mine], now[new_at]) and (got[:6] == 0).all() and (got[6 + 2 * new:] == 0).all()
        q = torch.randn(n, 4, D, generator=_gen(9), device="cuda").to(kind)
        out = torch.full_like(q, 7.0)
        b.cache.attend(q, b.table, b.seq_len, start, max_q=new, out=out)
        want = b.cache.attend(q[mine], b.table, b.seq_len, start - 6, max_q=new)
        assert torch.equal(out[mine], want) and (out[:6] == 7).all() and (out[6 + 2 * new:] == 7).all()
        torch.cuda.synchronize()
        assert b.cache.status() == 0


@pytest.mark.parametrize("D,H,new", [(64, 16, 17), (128, 16, 24), (64, 16, 32), (128, 64, 5), (64, 64, 6), (64, 64, 8), (128, 64, 8)])
def test_many_short_sequences_of_several_rows(D, H, new):
    """17 to 32 rows a key/value head in more heads and sequences than four an SM: several items for one sequence and head in
    the kernel for few rows.  Lengths from none; sequences with fewer rows than the most, or none."""
    Hkv = 16
    lens = [(53 * i) % 211 for i in range(39)] + [700]
    rows = [min(n, new if i % 3 else (7 * i) % (new + 1)) for i, n in enumerate(lens)]
    rows[1] = min(lens[1], new)
    assert max(rows) == new and 16 < new * (H // Hkv) <= 32 and len(lens) * Hkv > 4 * 148
    b = Batch(lens, Hkv, D, 32, seed=D + H + new)
    b.check(H, rows, max_q=new)
    b.check(H, rows, max_q=new, max_kv=max(lens), window=70)
    b.check(H, rows, max_q=new, window=9)
    b.check(H, rows, max_q=new, causal=False, scale=-0.3)


@pytest.mark.parametrize("H,Hkv,D", [(8, 2, 64), (4, 4, 128)])
def test_a_prompt_among_single_tokens(H, Hkv, D):
    """One prompt beside 31 sequences of one token behind some 4000 positions, one of them long: the most rows of a sequence
    choose the kernel for all."""
    lens = [512] + [3900 + 13 * i for i in range(30)] + [20000]
    new = [512] + [1] * 31
    b = Batch(lens, Hkv, D, 64, seed=H)
    b.check(H, new, max_q=512)
    b.check(H, new, max_q=512, max_kv=20000, window=1000)


@pytest.mark.parametrize("D,H,new,qmul", [(64, 8, 1, 40.0), (128, 4, 1, 40.0), (128, 8, 3, 40.0), (128, 4, 1, 4.0), (64, 12, 2, 12.0)])
def test_scores_of_few_rows_carry_no_rounding_of_keys(D, H, new, qmul):
    """The kernel for few rows multiplies q (exact in fp16) with the codes and adds in fp32: a score is off by at most
    (4 D + 8) u of scale sum |q| (|base| + 15 step) -- fp32 sums of D products of which the tensor cores cut each, the sums of q in
    two fp16 terms, two products and one sum more -- in the place of u16 scale sum |q k|.  The rest as in test_serving_gpu."""
    import torch
    Hkv = 2
    b = Batch([777, 130], Hkv, D, 64, seed=D)
    rows = 2 * new
    q = (torch.randn(rows, H, D, generator=_gen(11), device="cuda") * qmul).bfloat16()
    start = torch.tensor([0, new, rows], dtype=torch.int32, device="cuda")
    out = b.cache.attend(q, b.table, b.seq_len, start, max_q=new, causal=False).double().cpu().numpy()
    scale = 1 / math.sqrt(D)
    want, size, _ = b.plain(q, [new, new], False, 0, scale)
    per_group = np.abs(q.double().cpu().numpy()).reshape(rows, H, D // 32, 32).sum(-1)
    amp = []
    for s, k in enumerate(b.k):
        g = k.reshape(*k.shape[:-1], D // 32, 32)
        lo, hi = g.min(-1), g.max(-1)
        reach = np.repeat(np.abs(lo) + (hi - lo) * (1 + 2.0 ** -9), H // Hkv, axis=1)             # [positions, heads, groups]
        amp.append(np.einsum("ihg,jhg->ihj", per_group[s * new:(s + 1) * new], reach).max(-1) * scale)
    d = (4 * D + 8) * U * np.concatenate(amp)[..., None]
    tol = (2 * d + 3 * U16 + 2 * 777 * U) * size + U8 * np.abs(want)
    err = np.abs(out - want) / tol
    assert err.max() <= 1, f"worst {err.max():.3g} of the tolerance"


def _stalled(call, status):
    """A call whose input is withheld ends by itself, says TSVD_E_TIMEOUT once, and leaves what follows as it was."""
    import time

    import torch
    from paper_2308_07641_b200 import binding
    want = call(0)
    torch.cuda.synchronize()
    assert status() == 0
    t0 = time.perf_counter()
    call(binding.TSVD_FLAG_TEST_STALL)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 < 5.0
    assert status() == binding.TSVD_E_TIMEOUT and status() == 0
    for _ in range(2):
        assert torch.equal(call(0), want)
    torch.cuda.synchronize()
    assert status() == 0


@pytest.mark.parametrize("B,N,M", [(1, 4096, 640), (40, 300, 200), (600, 512, 40000)])
def test_layer_waits_give_up(B, N, M):
    """A few tokens (clusters), a single block's contraction, and blocks that walk over several tiles."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, quantize
    layer = Int8Linear(*quantize(torch.randn(M, N, generator=_gen(M), device="cuda")))
    x = torch.randn(B, N, generator=_gen(B), device="cuda").bfloat16()
    _stalled(lambda flags: layer(x, flags=flags), layer.status)


@pytest.mark.parametrize("lens,new,H,Hkv,D", [([50], [1], 2, 2, 64), ([9000, 70], [1, 1], 8, 2, 128), ([400, 300], [3, 3], 16, 4, 64),
                                              ([600], [300], 4, 2, 128), ([3000], [40], 4, 4, 64)])
def test_attention_waits_give_up(lens, new, H, Hkv, D):
    """Blocks apart, parts that blocks add up, items of sixteen rows; many rows, and with positions shared by blocks."""
    import torch
    b = Batch(lens, Hkv, D, 64, seed=H)
    q = torch.randn(sum(new), H, D, generator=_gen(5), device="cuda").bfloat16()
    start = torch.tensor([0] + [sum(new[:i + 1]) for i in range(len(new))], dtype=torch.int32, device="cuda")
    _stalled(lambda flags: b.cache.attend(q, b.table, b.seq_len, start, max_q=max(new), flags=flags), b.cache.status)


def test_binding_entry_points():
    """The one-to-one functions of `binding`, with raw pointers on the default stream, against the torch front."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, KV4Cache, binding, dequantize, quantize
    g = _gen(21)
    x = torch.randn(9, 200, generator=g, device="cuda")
    q, scale = quantize(x)
    y = dequantize(q, scale)
    q2, scale2, y2 = torch.zeros_like(q), torch.zeros_like(scale), torch.zeros_like(y)
    layer = Int8Linear(q, scale)
    out = layer(x)
    out2 = torch.zeros_like(out)
    cache, other = KV4Cache(2, 64, 4, 16), KV4Cache(2, 64, 4, 16)
    k, v = (torch.randn(3, 2, 64, generator=g, device="cuda") for _ in range(2))
    a = torch.randn(3, 4, 64, generator=g, device="cuda").bfloat16()
    table = torch.arange(3, dtype=torch.int32, device="cuda").view(3, 1)
    n, start = torch.ones(3, dtype=torch.int32, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    cache.append(k, v, table, n, start)
    rk, rv = cache.read(3, table, n, start)
    want = cache.attend(a, table, n, start, max_q=1)
    rk2, rv2, got = torch.zeros_like(rk), torch.zeros_like(rv), torch.zeros_like(want)
    torch.cuda.synchronize()
    F32, BF16, stream = binding.TSVD_F32, binding.TSVD_BF16, torch.cuda.current_stream().cuda_stream
    binding.tsvd_quantize(x.data_ptr(), F32, 9, 200, 200, q2.data_ptr(), q2.stride(0), scale2.data_ptr(), stream)
    binding.tsvd_dequantize(q.data_ptr(), q.stride(0), scale.data_ptr(), 9, 200, y2.data_ptr(), F32, 200, stream)
    binding.tsvd_i8_forward(layer.handle, x.data_ptr(), 200, 0, out2.data_ptr(), 9, 9, F32, 0, stream)
    batch = (table.data_ptr(), 1, n.data_ptr(), start.data_ptr(), 3, 3)
    binding.tsvd_kv4_append(other.handle, k.data_ptr(), 128, v.data_ptr(), 128, F32, *batch, stream)
    binding.tsvd_kv4_read(other.handle, rk2.data_ptr(), 128, rv2.data_ptr(), 128, F32, *batch, stream)
    binding.tsvd_kv4_attend(other.handle, a.data_ptr(), 256, got.data_ptr(), 256, 4, BF16, *batch, 1, 0, 0.125, 0, binding.TSVD_FLAG_CAUSAL,
                            stream)
    torch.cuda.synchronize()
    for mine, theirs in ((q2, q), (scale2, scale), (y2, y), (out2, out), (rk2, rk), (rv2, rv), (got, want)):
        assert torch.equal(mine, theirs)
    assert binding.tsvd_i8_info(layer.handle)["M"] == 9 and binding.tsvd_i8_info(layer.handle)["N"] == 200
    assert binding.tsvd_kv4_info(cache.handle) == {"n_kv_heads": 2, "head_dim": 64, "page_tokens": 16, "n_pages": 4, "pool_bytes": 4 * 2 * 20 * 64}
    assert binding.tsvd_i8_last_status(layer.handle) == 0 and binding.tsvd_kv4_last_status(other.handle) == 0
