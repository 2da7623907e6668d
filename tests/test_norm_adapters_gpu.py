"""Root-mean-square norm and low-rank adapters against plain implementations in 64 bits.

Tolerances (u8 = 2^-8 and u = 2^-24 are the unit roundoffs of bf16 and fp32):
  norm        h and the 8-bit values: equal, their definition is elementwise in fp32.  The sum of squares of n numbers, all
              positive: a chain of at most n / 32 + 20 additions, each off by u, and n squares, off by u; rho half of that and 4 u
              for its own operations: e = (n / 64 + 15) u.  scale: e + 3 u relative; y: e + 3 u relative, and its type's rounding
  adapters    products of bf16 numbers are exact in fp32; a step of the tensor core adds 16 of them to a sum and is taken to be
              off by at most 2^-21 of the sum of the magnitudes (17 addends cut two bits below fp32's last).  z = A x: at most
              N / 16 + 60 steps and additions (three times the steps for fp32 x, whose terms are exact), S1 = 2^-21 steps sum |a x|;
              its factor 4 u |z|; as two terms 2^-16 |z| (bf16 results).  out: those times |B|, rank / 16 * 3 + 1 steps of
              2^-21 sum |b z|, 2 u |out| and the result's rounding
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U, U8, STEP = 2.0 ** -24, 2.0 ** -8, 2.0 ** -21


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


# ---- the norm ----------------------------------------------------------------------------------------------------------


def _plain_rows8(h, w):
    """Values and their largest product of each row, elementwise in fp32 on the host: the definition."""
    t = h.float().cpu().numpy() * w.float().cpu().numpy()[None, :]
    a = np.abs(t).max(axis=1)
    inv = np.zeros_like(a)
    np.divide(np.float32(1), a, out=inv, where=a >= np.float32(2.0 ** -100))
    inv = inv * np.float32(127)
    return np.rint(t * inv[:, None]).astype(np.int8), a


def _check_norm(x, w, eps, r):
    import torch
    from paper_2308_07641_b200 import rms_norm, rms_norm_quantize
    y, q = rms_norm(x, w, eps, residual=r), rms_norm_quantize(x, w, eps, residual=r)
    h = x
    if r is not None:
        h = (x.float() + r.float()).to(x.dtype)
        assert torch.equal(y[1], h) and torch.equal(q[2], h) and y[1].dtype == x.dtype
        y = y[0]
    q, scale = q[:2]
    n = x.shape[1]
    d, e = h.double(), (n / 64 + 15) * U
    rho = 1 / (d.square().mean(1, keepdim=True) + eps).sqrt()
    want = d * rho * w.double()
    tol = (e + 3 * U + (U8 if x.dtype == torch.bfloat16 else U)) * want.abs() + 1e-38
    assert y.dtype == x.dtype and ((y.double() - want).abs() <= tol).all()
    want_q, a = _plain_rows8(h, w)
    assert np.array_equal(q.cpu().numpy(), want_q)
    want_s = a.astype(np.float64) / 127 * rho[:, 0].cpu().numpy()
    assert (np.abs(scale.double().cpu().numpy() - want_s) <= (e + 3 * U) * want_s + 1e-44).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 7, 1, 0), (3, 64, 0, 0), (5, 100, 12, 0), (2, 129, 7, 1), (4, 1001, 0, 3),
                                                 (3, 4096, 0, 0), (2, 4097, 0, 0), (1, 8192, 0, 0), (3, 8200, 8, 0), (2, 16384, 0, 0),
                                                 (2, 20000, 8, 0), (1, 70001, 0, 0), (700, 256, 0, 0), (2500, 40, 0, 0), (2049, 513, 7, 5)])
def test_norm(dtype, rows, cols, pad, shift):
    import torch
    g = _gen(rows * 1000 + cols)
    make = lambda: torch.randn(rows * (cols + pad) + shift, generator=g, device="cuda").mul_(3).to(_dtype(dtype))[shift:].view(  # noqa: E731
        rows, cols + pad)[:, :cols]
    x, r = make(), make()
    if rows > 2:
        x[1] = 0
        x[2] *= 1e-3
    w = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda"))
    _check_norm(x, w, 1e-5, None)
    _check_norm(x, w.bfloat16(), 1e-6, r)


def test_norm_weights_anywhere():
    import torch
    g = _gen(4)
    x, w = torch.randn(6, 512, generator=g, device="cuda"), torch.randn(520, generator=g, device="cuda")
    _check_norm(x, w[3:515], 1e-6, None)
    _check_norm(x.bfloat16(), w[1:513], 1e-6, x.flip(0).bfloat16())


@pytest.mark.parametrize("cols", [300, 40000])
def test_norm_extreme_rows(cols):
    import torch
    from paper_2308_07641_b200 import dequantize, rms_norm, rms_norm_quantize
    x = torch.randn(7, cols, generator=_gen(1), device="cuda")
    x[0] *= 1e30                       # squares beyond fp32
    x[1] *= 1e-30                      # squares below it: eps decides
    x[2] = 0
    x[3, 5] = float("inf")
    x[4, cols - 1] = float("nan")
    x[5] = torch.where(torch.arange(cols, device="cuda") == 7, 3e38, 0.0)
    w = torch.ones(cols, device="cuda")
    fine = [0, 1, 2, 5, 6]
    y, (q, scale) = rms_norm(x, w, 1e-6), rms_norm_quantize(x, w, 1e-6)
    d = x.double()
    want = d / (d.square().mean(1, keepdim=True) + 1e-6).sqrt()
    e = (cols / 64 + 15) * U
    assert ((y.double() - want)[fine].abs() <= (e + 4 * U) * want[fine].abs() + 2.0 ** -149).all()
    step = scale.double()[:, None]
    back = dequantize(q, scale).double()
    # half a step, and what the scale is off by; a row below 2^-100 is zeros
    assert ((back - want)[[0, 2, 5, 6]].abs() <= 0.5 * step[[0, 2, 5, 6]] * (1 + 300 * (e + 4 * U)) + 1e-30).all()
    assert not torch.isfinite(y[3]).all() and not torch.isfinite(y[4]).all()
    assert not torch.isfinite(scale[3]) and not torch.isfinite(scale[4]) and torch.isfinite(scale[fine]).all()


def test_norm_in_place_through_the_binding():
    """h over the residual or over x, y over x: each number is read before it is written."""
    import torch
    from paper_2308_07641_b200 import binding, rms_norm
    for cols in (256, 4096, 33000):
        g = _gen(cols)
        x, r = (torch.randn(5, cols, generator=g, device="cuda").bfloat16() for _ in range(2))
        w = torch.randn(cols, generator=g, device="cuda")
        want_y, want_h = rms_norm(x, w, 1e-6, residual=r)
        plain_y = rms_norm(x, w, 1e-6)
        stream = torch.cuda.current_stream().cuda_stream
        for over in ("r", "x"):
            a, b, y = x.clone(), r.clone(), torch.empty_like(x)
            h = b if over == "r" else a
            binding.tsvd_rms_norm(a.data_ptr(), 1, 5, cols, cols, b.data_ptr(), cols, h.data_ptr(), cols, w.data_ptr(), 0, 1e-6, y.data_ptr(), cols,
                                  0, 0, 0, stream)
            assert torch.equal(h, want_h) and torch.equal(y, want_y)
        a = x.clone()
        binding.tsvd_rms_norm(a.data_ptr(), 1, 5, cols, cols, 0, 0, 0, 0, w.data_ptr(), 0, 1e-6, a.data_ptr(), cols, 0, 0, 0, stream)
        assert torch.equal(a, plain_y)


def test_norm_feeds_the_layer():
    """The 8-bit rows with their scales are what Int8Linear takes, and nothing is lost on the way."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, dequantize, quantize, rms_norm_quantize
    g = _gen(7)
    x, w = torch.randn(70, 640, generator=g, device="cuda").bfloat16(), torch.randn(640, generator=g, device="cuda")
    layer = Int8Linear(*quantize(torch.randn(200, 640, generator=g, device="cuda")))
    q, scale = rms_norm_quantize(x, w)
    y = layer(q, scale)
    back = layer(q, torch.ones_like(scale))
    want = back.double() * scale.double()[:, None]
    assert ((y.double() - want).abs() <= 3 * U * want.abs()).all()
    assert dequantize(q, scale).shape == x.shape
    assert rms_norm_quantize(x[:0], w)[0].shape == (0, 640)


# ---- adapters ------------------------------------------------------------------------------------------------------------


class Adapters:
    def __init__(self, N, M, ranks, seed=0, max_rank=None, dtype="bf16", extra=0):
        import torch
        from paper_2308_07641_b200 import LowRankAdapters
        g = _gen(seed + 5)
        self.N, self.M = N, M
        self.h = LowRankAdapters(N, M, max_rank or max(max(ranks), 1), len(ranks) + extra)
        self.A, self.B, self.c = [], [], []
        for s, r in enumerate(ranks):
            a = (torch.randn(max(r, 1), N + 3, generator=g, device="cuda") / N ** 0.5).to(_dtype(dtype))[:, 1:N + 1]
            b = torch.randn(M, max(r, 1) + 2, generator=g, device="cuda").to(_dtype(dtype))[:, 2:]
            c = 0.5 + 0.25 * s
            if r:
                self.h.set(s, a, b, c)
            self.A.append(a.bfloat16().double()[:r])
            self.B.append(b.bfloat16().double()[:, :r])
            self.c.append(c)

    def check(self, x, base, slots, new, x_scale=None, none=-1, **kw):
        """slots: of each sequence; new: their rows (None: one each)."""
        import torch
        start = None if new is None else torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        out = self.h(x, base, torch.tensor(slots, dtype=torch.int32, device="cuda"), start, x_scale=x_scale, **kw)
        rows = [s for s, n in zip(slots, new or [1] * len(slots)) for _ in range(n)]
        assert len(rows) == x.shape[0]
        d = x.double() * (1 if x_scale is None else x_scale.double()[:, None])
        want = torch.zeros(x.shape[0], self.M, dtype=torch.float64, device="cuda") if base is None else base.double().clone()
        tol = torch.zeros_like(want)
        bf16 = out.dtype == torch.bfloat16
        rows = torch.tensor(rows)
        for s in sorted(set(rows.tolist())):
            if s < 0 or s >= len(self.A) or self.A[s].shape[0] == 0:
                continue
            at = (rows == s).to("cuda")
            xs, A, B, c = d[at], self.A[s], self.B[s], self.c[s]
            z, reach = xs @ A.T, xs.abs() @ A.abs().T
            steps = (3 if x.dtype == torch.float32 else 1) * self.N / 16 + 60
            dz = STEP * steps * reach + (4 * U + (2.0 ** -16 if bf16 else 0)) * z.abs()
            want[at] += c * (z @ B.T)
            tol[at] = c * (dz @ B.abs().T + (A.shape[0] / 16 * 3 + 4) * STEP * (z.abs() @ B.abs().T))
        tol = tol * 1.01 + 2 * U * want.abs() + (U8 if bf16 else U) * want.abs() + 1e-30
        adapted = ((rows >= 0) & (rows < len(self.A))).to("cuda")
        err = (out.double() - want).abs() / tol
        assert err.max() <= 1, f"worst {float(err.max()):.3g} of the tolerance"
        if base is not None:
            assert torch.equal(out[~adapted], base[~adapted])
        return out


def _rows(kind, n, N, g, pad=0):
    """x (with padding behind each row) and its scales."""
    import torch
    x = torch.randn(n, N + pad, generator=g, device="cuda")
    if kind == "i8":
        return (x * 40).round().clamp(-127, 127).to(torch.int8)[:, :N], torch.rand(n, generator=g, device="cuda") + 0.1
    return x.to(_dtype(kind))[:, :N], None


CASES = [
    # N, M, ranks, slots, rows of each sequence (None: one)
    (1, 1, [1], [0], None), (32, 64, [16], [0], None), (64, 64, [4, 16], [1, 0, -1, 1], None), (100, 70, [3, 8], [0, 1], [1, 3]),
    (1001, 770, [9, 4, 2], [2, 0, -1, 1, 0], [49, 7, 1, 0, 20]), (4096, 512, [16, 8, 64, 1], [i % 5 - 1 for i in range(64)], None),
    (257, 4096, [16] * 20, [(7 * i) % 20 for i in range(33)], None), (512, 300, [33, 128, 17], [0, 1, 2, 1], [5, 40, 17, 1]),
    (640, 1030, [64], [0], [300]), (2048, 640, [16, 32], [0, 1, -1, 0], [500, 77, 30, 600]), (333, 200, [48, 5], [0, 1] * 40, [17] * 80),
    (96, 129, [112], [0, 0, -1], [15, 2, 9]), (8200, 64, [8], [0, 0], None), (64, 8200, [8, 24], [1, 0, 1], [1, 70, 1]),
    (768, 768, [8] * 40, list(range(40)), [3] * 40), (128, 256, [16], [-1, -1], [2, 1]), (300, 130, [20, 90], [0, 1, 0], [400, 700, 30]),
]


@pytest.mark.parametrize("N,M,ranks,slots,new", CASES)
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f32", "f32"), ("i8", "f32"), ("bf16", "f32"), ("i8", "bf16")])
def test_adapters(N, M, ranks, slots, new, kind, out):
    import torch
    g = _gen(N + M)
    a = Adapters(N, M, ranks, dtype="f32" if kind == "f32" else "bf16")
    n = len(slots) if new is None else sum(new)
    for pad, shift in ((-N % 16, 0), (3, 5)):                # aligned rows, and others
        x, x_scale = _rows(kind, n, N, g, pad)
        base = torch.randn(n, M + (-M % 8 if shift == 0 else 1), generator=g, device="cuda").to(_dtype(out))[:, :M]
        got = a.check(x, base, slots, new, x_scale)
        again = a.h(x, base, torch.tensor(slots, dtype=torch.int32, device="cuda"),
                    None if new is None else torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda"), x_scale=x_scale)
        assert torch.equal(got, again)
    if kind == "i8":
        a.check(x, base, slots, new, None)
    if (kind == "bf16") == (out == "bf16"):
        a.check(x, None, slots, new, x_scale)
    assert a.h.status() == 0


MANY = [
    # N, M, ranks, slots, rows of each sequence: 600 rows or so, 64 a sequence as a mean (ranks above 48: 200, 32); tiles of up to 128 rows,
    # stages of 64 columns
    (32, 64, [16], [0], [512]), (64, 1, [1], [0], [513]), (96, 130, [128, 3], [0, 1, 0], [129, 255, 128]), (8, 72, [8, 8], [1, 0], [127, 640]),
    (1001, 770, [9, 64, 33], [2, 0, -1, 1, 0, 1], [349, 1, 100, 0, 255, 90]), (4096, 192, [16, 100], [0, 1, -1, 0, 1], [1, 2, 600, 5, 900]),
    (520, 328, [64] * 8, list(range(8)), [64, 65, 63, 1, 127, 128, 129, 60]), (200, 4100, [32], [-1, 0, -1], [300, 256, 44]),
    (640, 640, [0, 0, 20], [0, 1], [400, 200]), (328, 2100, [64, 50], [0, 1, 0], [66, 100, 51]), (264, 200, [128, 70], [1, 0, 1, -1], [40, 31, 90, 40]),
]


@pytest.mark.parametrize("N,M,ranks,slots,new", MANY)
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f32", "f32"), ("i8", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("i8", "bf16")])
def test_adapters_many_rows(N, M, ranks, slots, new, kind, out):
    """Whole sequences in tiles: rows of nobody ahead, behind and between stay as they were; in place; no base; x that cannot be copied
    sixteen bytes at a time."""
    import torch
    g = _gen(N + M + len(new))
    a = Adapters(N, M, ranks, dtype="f32" if kind == "f32" else "bf16")
    n = sum(new)
    for pad in (-N % 16, 1 - N % 2):
        x, x_scale = _rows(kind, n, N, g, pad)
        base = torch.randn(n, M + -M % 8, generator=g, device="cuda").to(_dtype(out))[:, :M]
        want = a.check(x, base, slots, new, x_scale)
        over = base.clone()
        start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        ids = torch.tensor(slots, dtype=torch.int32, device="cuda")
        a.h(x, over, ids, start, x_scale=x_scale, out=over)
        assert torch.equal(over, want)
        start = start.clamp(3, n - 2)                          # (borders ascend)
        left = torch.full((n + 1, M + 1), 7.0, device="cuda").to(_dtype(out))
        a.h(x, base, ids, start, x_scale=x_scale, out=left[:n, :M])
        assert (left[:3] == 7).all() and (left[n - 2:] == 7).all() and (left[:, M] == 7).all()
        assert torch.isfinite(left).all()
        if (kind == "bf16") == (out == "bf16"):
            a.check(x, None, slots, new, x_scale)
    assert a.h.status() == 0


def test_adapters_many_rows_keep_to_themselves():
    """What is not finite in a row or an adapter stays with it, in tiles that other rows share too."""
    import torch
    g = _gen(18)
    a = Adapters(328, 200, [8, 8, 20])
    a.h.set(1, torch.full((8, 328), float("nan"), device="cuda"), torch.full((200, 8), float("inf"), device="cuda"))
    x, base = torch.randn(700, 328, generator=g, device="cuda").bfloat16(), torch.randn(700, 200, generator=g, device="cuda").bfloat16()
    x[3], x[517] = float("nan"), float("inf")
    new, slots = [150, 250, 300], [0, 1, 2]
    start = torch.tensor([0, 150, 400, 700], dtype=torch.int32, device="cuda")
    out = a.h(x, base, torch.tensor(slots, dtype=torch.int32, device="cuda"), start)
    ok = torch.ones(700, dtype=torch.bool, device="cuda")
    ok[150:400] = ok[3] = ok[517] = False
    assert torch.isfinite(out[ok]).all() and not torch.isfinite(out[~ok]).any()
    x[3] = x[517] = 0
    clean = a.check(x[:150], base[:150], [0], [150])
    assert ((clean.double() - out[:150].double()).abs()[ok[:150]] <= 4 * U8 * clean.double().abs()[ok[:150]] + 1e-2).all()
    a.h.clear(1)
    again = a.check(x, base, [0, -1, 2], new)
    assert torch.equal(again[150:400], base[150:400])


def test_adapters_many_rows_move_under_a_graph():
    """The number of tiles is counted on the device: borders that move, also beyond the rows, and slots that are not there."""
    import torch
    from paper_2308_07641_b200 import binding
    g = _gen(19)
    a = Adapters(256, 320, [24, 64, 5])
    n = 700
    x, base = torch.randn(n, 256, generator=g, device="cuda").bfloat16(), torch.randn(n, 320, generator=g, device="cuda").bfloat16()
    start = torch.tensor([0, 128, 256, 384, 512, 640, 700], dtype=torch.int32, device="cuda")
    slots = torch.tensor([0, 1, 2, 0, 1, 2], dtype=torch.int32, device="cuda")
    a.h.reserve(n)
    out = torch.empty_like(base)
    a.h(x, base, slots, start, out=out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.h(x, base, slots, start, out=out)
    for new, ids in (([128, 128, 128, 128, 128, 60], [0, 1, 2, 0, 1, 2]), ([129, 1, 129, 1, 129, 311], [2, 1, 0, -1, 1, 0]),
                     ([0, 0, 700, 0, 0, 0], [0, 1, 1, 2, 0, 1]), ([1, 1, 1, 1, 1, 695], [0, 1, 2, 0, -1, 2]), ([117] * 5 + [115], [-1] * 6)):
        start.copy_(torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32))
        slots.copy_(torch.tensor(ids, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        assert torch.equal(out, a.check(x, base, ids, new))
    # beyond the rows: cut off; slots that are not there: base, and a status
    want = a.check(x, base, [0, 1, 2, -1, -1, 0], [100, 100, 100, 100, 100, 200])
    start.copy_(torch.tensor([-9, 100, 200, 300, 400, 500, 2 ** 31 - 1], dtype=torch.int32))
    slots.copy_(torch.tensor([0, 1, 2, 3, -2 ** 31, 0], dtype=torch.int32))
    assert a.h.status() == 0
    graph.replay()
    assert torch.equal(out, want)
    assert a.h.status() == binding.TSVD_E_INDEX and a.h.status() == 0


@pytest.mark.parametrize("rank", [16, 32, 64, 128])
def test_adapters_reserved_rows_need_no_memory(rank):
    """A first call under capture, whichever way it takes: nothing is allocated after reserve."""
    import torch
    g = _gen(rank)
    a = Adapters(4096, 4096, [rank, rank])
    a.h.reserve(300)
    for n, new in ((300, [100, 200]), (300, [1] * 300), (200, [150, 50]), (40, [40]), (1, [1])):
        x, base = (torch.randn(n, 4096, generator=g, device="cuda").bfloat16() for _ in range(2))
        slots = torch.tensor([i % 2 for i in range(len(new))], dtype=torch.int32, device="cuda")
        start = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = a.h(x, base, slots, start)
        graph.replay()
        assert torch.equal(out, a.check(x, base, slots.tolist(), new))


def test_adapters_in_place_and_bounds():
    """out is base; rows of an out with padding; rows of no sequence, and what lies beside the rows, stay as they were."""
    import torch
    g = _gen(3)
    a = Adapters(200, 100, [8, 16])
    x = torch.randn(20, 200, generator=g, device="cuda").bfloat16()
    store = torch.randn(22, 120, generator=g, device="cuda").bfloat16()
    base = store[1:21, 8:108]
    want = a.check(x, base.clone(), [0, -1, 1], [7, 5, 8])
    before = store.clone()
    slots = torch.tensor([0, -1, 1], dtype=torch.int32, device="cuda")
    a.h(x, base, slots, torch.tensor([0, 7, 12, 20], dtype=torch.int32, device="cuda"), out=base)
    assert torch.equal(base, want)
    base.copy_(before[1:21, 8:108])
    assert torch.equal(store, before)
    # rows 0, 1 and 15 .. 19 belong to nobody
    out = torch.full((20, 100), 7.0, device="cuda").bfloat16()
    a.h(x, base, slots, torch.tensor([2, 7, 12, 15], dtype=torch.int32, device="cuda"), out=out)
    assert (out[:2] == 7).all() and (out[15:] == 7).all() and torch.equal(out[2:7], want[2:7]) and torch.equal(out[7:12], base[7:12])
    assert torch.equal(out[12:15], want[12:15])


def test_adapters_keep_to_themselves():
    """What is not finite in a row or an adapter stays with it."""
    import torch
    g = _gen(8)
    a = Adapters(300, 200, [8, 8, 20])
    bad_A = torch.full((8, 300), float("nan"), device="cuda")
    a.h.set(1, bad_A, torch.full((200, 8), float("inf"), device="cuda"))
    x, base = torch.randn(40, 300, generator=g, device="cuda").bfloat16(), torch.randn(40, 200, generator=g, device="cuda").bfloat16()
    x[3] = float("nan")
    x[17] = float("inf")
    slots = [i % 3 for i in range(40)]
    out = a.h(x, base, torch.tensor(slots, dtype=torch.int32, device="cuda"))
    fine = [i for i in range(40) if i % 3 != 1 and i not in (3, 17)]
    assert torch.isfinite(out[fine]).all() and not torch.isfinite(out[[i for i in range(40) if i not in fine]]).any()
    keep = [i for i in fine]
    assert torch.equal(a.check(x[keep], base[keep], [slots[i] for i in keep], None), out[keep])


def test_adapters_set_clear_and_slots_out_of_range():
    import torch
    from paper_2308_07641_b200 import binding
    g = _gen(9)
    a = Adapters(128, 96, [8, 0, 4], max_rank=16, extra=1)
    x, base = torch.randn(6, 128, generator=g, device="cuda"), torch.randn(6, 96, generator=g, device="cuda")
    a.check(x, base, [0, 1, 2, 3, -1, 0], None)                 # empty slots add nothing
    assert a.h.status() == 0
    out = a.h(x, base, torch.tensor([0, 4, -2, 2 ** 31 - 1, -2 ** 31, 2], dtype=torch.int32, device="cuda"))
    assert torch.equal(out[1:5], base[1:5])
    torch.cuda.synchronize()
    assert a.h.status() == binding.TSVD_E_INDEX and a.h.status() == 0
    # another adapter, of another rank, into a used slot, in the stream's order
    for r in (16, 3):
        A, B = torch.randn(r, 128, generator=g, device="cuda"), torch.randn(96, r, generator=g, device="cuda")
        a.h.set(0, A, B, -2.0)
        a.A[0], a.B[0], a.c[0] = A.bfloat16().double(), B.bfloat16().double(), 2.0
        A.zero_()                                              # (a copy was taken)
        a.B[0] = -a.B[0]
        a.check(x, base, [0] * 6, None)
    a.h.clear(0)
    assert torch.equal(a.h(x, base, torch.zeros(6, dtype=torch.int32, device="cuda")), base)
    assert a.h.status() == 0 and binding.tsvd_adapters_info(a.h.handle)["n_slots"] == 4


def test_adapters_no_rows():
    import torch
    a = Adapters(64, 64, [4])
    e = torch.empty(0, 64, device="cuda")
    assert a.h(e, e, torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 64)


def test_adapters_change_under_a_graph():
    """Slots, rows and sequence borders are read on the device; a graph captured before the scratch grew stays valid, beside another."""
    import torch
    a = Adapters(700, 500, [8, 16, 3])
    g = _gen(12)
    x, base = torch.randn(30, 700, generator=g, device="cuda").bfloat16(), torch.randn(30, 500, generator=g, device="cuda").bfloat16()
    slots, start = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.tensor([0, 10, 20, 30], dtype=torch.int32, device="cuda")
    one = torch.zeros(30, dtype=torch.int32, device="cuda")
    a.h.reserve(30)
    out, out1 = torch.empty_like(base), torch.empty_like(base)
    graphs = []
    for s, q, o in ((slots, start, out), (one, None, out1)):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.h(x, base, s, q, out=o)
        graphs.append(graph)
    big = torch.randn(2000, 700, generator=g, device="cuda").bfloat16()
    a.h(big, None, torch.zeros(2000, dtype=torch.int32, device="cuda"))        # grows
    for pick, ends in (([0, 1, 2], [0, 10, 20, 30]), ([2, -1, 0], [0, 1, 25, 30])):
        slots.copy_(torch.tensor(pick))
        start.copy_(torch.tensor(ends))
        one.copy_(torch.tensor([i % 3 for i in range(30)]))
        x.normal_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, a.check(x, base, pick, [b - a_ for a_, b in zip(ends, ends[1:])]))
        assert torch.equal(out1, a.check(x, base, one.tolist(), None))


def test_norm_and_adapters_on_another_stream():
    """In a chain, each a programmatic dependent of the one ahead: the same bits as one by one."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, quantize, rms_norm_quantize
    g = _gen(15)
    a = Adapters(512, 768, [16, 8, 4])
    layer = Int8Linear(*quantize(torch.randn(768, 512, generator=g, device="cuda")))
    w = torch.randn(512, generator=g, device="cuda")
    layer.reserve(600, "i8")
    a.h.reserve(600)
    for n in (1, 5, 40, 600):
        x, r = (torch.randn(n, 512, generator=g, device="cuda").bfloat16() for _ in range(2))
        slots = torch.tensor([i % 4 - 1 for i in range(n)], dtype=torch.int32, device="cuda")
        wants = []
        h = r
        for _ in range(3):
            q, scale, h = rms_norm_quantize(x, w, residual=h)
            torch.cuda.synchronize()
            y = layer(q, scale)
            torch.cuda.synchronize()
            wants.append(a.h(q, y, slots, x_scale=scale))
            torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(4):
                h, got = r, []
                for _ in range(3):
                    q, scale, h = rms_norm_quantize(x, w, residual=h)
                    y = layer(q, scale)
                    got.append(a.h(q, y, slots, x_scale=scale, out=y))
                side.synchronize()
                for m, t in zip(got, wants):
                    assert torch.equal(m, t)
    assert layer.status() == 0 and a.h.status() == 0
