"""The adapters where a call meets its surroundings: waits that give up, results that are exact, whole sequences and mixed
batches, slots far larger than their adapters, a ternary projection beside them, the one-to-one functions of `binding`.
(Tolerances: test_norm_adapters_gpu.)"""
import numpy as np
import pytest

from tests.test_norm_adapters_gpu import Adapters, _dtype, _gen, _rows
from tests.test_serving_calls_gpu import _stalled

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2308_07641_b200 import build
    build.build()


def _start(new):
    import torch
    return torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("N,M,rank,new,kind,aligned", [
    (4096, 640, 64, [300, 300], "bf16", True), (4096, 640, 64, [300, 300], "i8", True), (1024, 640, 128, [150, 70], "f32", True),
    (128, 300, 128, [200, 70], "bf16", True), (64, 300, 70, [250], "f32", True), (128, 300, 128, [200, 70], "bf16", False),
    (512, 20000, 100, [130, 100], "bf16", True)])
def test_waits_give_up(N, M, rank, new, kind, aligned):
    """Both products, with more stages than places and with fewer (there the copying warps end as if nothing were wrong), contractions
    that clusters share; the second product alone (x that the first one cannot copy), and with many blocks of channels a block."""
    import torch
    g = _gen(N + rank)
    a = Adapters(N, M, [rank, 3])
    x, x_scale = _rows(kind, sum(new), N, g, -N % 16 if aligned else 1)
    base = torch.randn(sum(new), M, generator=g, device="cuda").to(_dtype("f32" if kind == "i8" else kind))
    slots, start = torch.tensor([0, 1][:len(new)], dtype=torch.int32, device="cuda"), _start(new)
    _stalled(lambda flags: a.h(x, base, slots, start, x_scale=x_scale, flags=flags), a.h.status)
    a.check(x, base, [0, 1][:len(new)], new, x_scale)


def test_forms_that_wait_for_nothing_take_no_notice():
    import torch
    from paper_2308_07641_b200 import binding
    g = _gen(2)
    a = Adapters(256, 192, [16])
    for n in (1, 40, 3000):
        x, base = torch.randn(n, 256, generator=g, device="cuda").bfloat16(), torch.randn(n, 192, generator=g, device="cuda").bfloat16()
        slots = torch.zeros(n, dtype=torch.int32, device="cuda")
        assert torch.equal(a.h(x, base, slots, flags=binding.TSVD_FLAG_TEST_STALL), a.h(x, base, slots))
    torch.cuda.synchronize()
    assert a.h.status() == 0


# ---- exact results -------------------------------------------------------------------------------------------------------

# (N, M, rank, rows of each sequence or None: one each, aligned): one launch; tiles of 8 and of 32 rows on mma.sync; whole sequences
FORMS = [(40, 70, 9, None, True), (4096, 1030, 64, [3, 5], True), (333, 200, 48, [17] * 8, False), (512, 300, 100, None, True),
         (600, 130, 128, [7, 1, 40], False), (257, 640, 30, [5] * 300, False), (512, 300, 33, [40] * 40, True), (329, 300, 17, [33] * 40, False),
         (2048, 4100, 33, [1] * 700, True), (640, 512, 16, [800, 700], True),
         (1001, 770, 48, [700, 3, 900], True), (520, 328, 128, [130, 129, 1], True), (200, 4100, 70, [64, 300], True), (328, 136, 100, [255, 70], False)]


@pytest.mark.parametrize("N,M,rank,new,aligned", FORMS)
@pytest.mark.parametrize("kind,out", [("f32", "f32"), ("i8", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_selected_numbers_come_through_exactly(N, M, rank, new, aligned, kind, out):
    """A holds one 1 a row and B one a row, so that a result is one number of x: bit for bit where the terms that fp32 x and A x are cut
    into add up to all 24 bits and every other product is 0; with base, one rounded fp32 addition on top.  8-bit x comes out times
    its scale, one fp32 product.  A row's numbers span 2^+-20 in size, so that a term lost or in a wrong place shows."""
    import torch
    from paper_2308_07641_b200 import LowRankAdapters
    g = _gen(N + M + rank)
    n = sum(new) if new else 41
    n_seq = len(new) if new else n
    take = torch.randint(0, N, (2, rank), generator=g, device="cuda")
    give = torch.randint(0, rank, (2, M), generator=g, device="cuda")
    h = LowRankAdapters(N, M, rank, 2)
    for s in range(2):
        h.set(s, torch.nn.functional.one_hot(take[s], N).to(_dtype("f32" if s else "bf16")), torch.nn.functional.one_hot(give[s], rank).to(
            _dtype("f32" if s else "bf16")), 1.0)
    x, x_scale = _rows(kind, n, N + (-N % 16 if aligned else 1 - N % 2), g)
    if kind != "i8":
        x = x * torch.exp2(torch.randint(-20, 21, x.shape, generator=g, device="cuda").float()).to(x.dtype)
    x = x[:, :N]
    slots = torch.arange(n_seq, dtype=torch.int32, device="cuda") % 2
    seq = torch.repeat_interleave(torch.arange(n_seq, device="cuda"), torch.tensor(new or [1] * n, device="cuda"))
    picked = take.gather(1, give)[seq % 2]                                # [rows, M]: which number of x
    want = x.float().gather(1, picked)
    if kind == "i8":
        want = want * x_scale[:, None]
    start = _start(new) if new else None
    got = h(x, None, slots, start, x_scale=x_scale) if (kind == "bf16") == (out == "bf16") else None
    if got is not None:
        assert torch.equal(got.float(), want)
    zero = torch.zeros(n, M, dtype=_dtype(out), device="cuda")
    assert torch.equal(h(x, zero, slots, start, x_scale=x_scale).float(), want)
    if out == "f32":
        base = torch.randn(n, M, generator=g, device="cuda")
        assert torch.equal(h(x, base, slots, start, x_scale=x_scale), base + want)
    torch.cuda.synchronize()
    assert h.status() == 0


# ---- batches of every kind ----------------------------------------------------------------------------------------------

# More rows than the one-launch form takes at these sizes, and sequences long enough for tiles of their own (64 rows a sequence, 32 with ranks above
# 48): both products on tcgen05 (fp32 x of one group of ranks: the first one from 4096 rows on), with one to eight groups of 16 ranks
WHOLE = [(32, 64, [16], [0], [1300]), (1001, 770, [9, 16, 3], [2, 0, -1, 1, 0], [349, 700, 100, 1, 255]), (520, 328, [32, 17], [0, 1, 0], [640, 127, 700]),
         (256, 2100, [48, 20], [1, 0, -1, 0], [66, 1100, 100, 51]), (640, 640, [64, 0, 50, 5], [0, 1, 2, 3], [400, 200, 129, 700]),
         (96, 130, [80, 3], [0, 1, 0], [129, 255, 128]), (264, 200, [96], [0, 0, -1], [100, 31, 129]), (72, 72, [112], [0, 0], [256, 1]),
         (328, 129, [128], [0], [193]), (72, 70, [16, 2], [0, 1], [4000, 200])]


@pytest.mark.parametrize("N,M,ranks,slots,new", WHOLE)
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("f32", "f32"), ("i8", "f32"), ("i8", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
def test_whole_sequences(N, M, ranks, slots, new, kind, out):
    """As wide as the ranks need; that the kernels on tcgen05 take the call is seen by their waits, which give up on request."""
    import torch
    from paper_2308_07641_b200 import binding
    g = _gen(N + M)
    a = Adapters(N, M, ranks, dtype="f32" if kind == "f32" else "bf16")
    x, x_scale = _rows(kind, sum(new), N, g, -N % 16)
    base = torch.randn(sum(new), M + -M % 8, generator=g, device="cuda").to(_dtype(out))[:, :M]
    want = a.check(x, base, slots, new, x_scale)
    over, ids = base.clone(), torch.tensor(slots, dtype=torch.int32, device="cuda")
    a.h(x, over, ids, _start(new), x_scale=x_scale, out=over)
    assert torch.equal(over, want)
    assert a.h.status() == 0
    a.h(x, base, ids, _start(new), x_scale=x_scale, flags=binding.TSVD_FLAG_TEST_STALL)
    torch.cuda.synchronize()
    assert a.h.status() == binding.TSVD_E_TIMEOUT
    assert torch.equal(a.check(x, base, slots, new, x_scale), want) and a.h.status() == 0


@pytest.mark.parametrize("tokens,prompts", [(63, [1024]), (15, [1024]), (31, [700, 1, 300]), (200, [64]), (7, [130])])
@pytest.mark.parametrize("N,M,ranks", [(1024, 1536, [16, 8, 64, 3]), (512, 700, [128, 5])])
def test_prompts_among_single_tokens(N, M, ranks, tokens, prompts):
    """What a serving loop submits; the form is chosen for the whole call."""
    import torch
    g = _gen(tokens)
    a = Adapters(N, M, ranks)
    new = [1] * (tokens // 2) + prompts + [1] * (tokens - tokens // 2)
    x, base = torch.randn(sum(new), N, generator=g, device="cuda").bfloat16(), torch.randn(sum(new), M, generator=g, device="cuda").bfloat16()
    a.check(x, base, [i % (len(ranks) + 1) - 1 for i in range(len(new))], new)
    assert a.h.status() == 0


@pytest.mark.parametrize("max_rank", [17, 64, 65, 128])
@pytest.mark.parametrize("new", [[1], [1] * 9, [5, 1, 17], [40] * 20, [300, 1000], [900, 1, 500]])
def test_slots_larger_than_their_adapters(max_rank, new):
    """The handle's largest rank chooses the form; the adapters in it are small, of unlike ranks, or not there."""
    import torch
    g = _gen(max_rank)
    a = Adapters(328, 200, [16, 1, 0, 9], max_rank=max_rank)
    for kind in ("bf16", "f32"):
        x, _ = _rows(kind, sum(new), 328, g)
        base = torch.randn(sum(new), 200, generator=g, device="cuda").to(_dtype(kind))
        a.check(x, base, [i % 5 - 1 for i in range(len(new))], new)
        a.check(x, base, [(i + 1) % 4 for i in range(len(new))], new)
    assert a.h.status() == 0


@pytest.mark.parametrize("new", [[1], [1] * 16, [3, 1, 28], [130, 70], [1500, 100]])
@pytest.mark.parametrize("rank", [8, 100])
def test_beside_a_ternary_layer(new, rank):
    """The ternary product's result is the base, in place, each call a programmatic dependent of the one ahead, on a side stream."""
    import torch
    from paper_2308_07641_b200 import TSVDLinear
    N, M, K = 512, 384, 256
    rng = np.random.default_rng(rank)
    layer = TSVDLinear(rng.integers(-1, 2, (M, K), dtype=np.int8), rng.random(K, dtype=np.float32) / 64, rng.integers(-1, 2, (K, N), dtype=np.int8))
    n, g = sum(new), _gen(rank)
    a = Adapters(N, M, [rank, 4])
    layer.reserve(n, "bf16")
    a.h.reserve(n)
    xs = [torch.randn(n, N, generator=g, device="cuda").bfloat16() for _ in range(6)]
    slots = [i % 3 - 1 for i in range(len(new))]
    ids, start = torch.tensor(slots, dtype=torch.int32, device="cuda"), _start(new)
    wants = []
    for x in xs:
        base = layer(x)
        torch.cuda.synchronize()
        wants.append(a.check(x, base, slots, new))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            outs = []
            for x in xs:
                y = layer(x)
                outs.append(a.h(x, y, ids, start, out=y))
            side.synchronize()
            assert all(torch.equal(y, want) for y, want in zip(outs, wants))
    assert a.h.status() == 0


def test_binding_entry_points():
    """The one-to-one functions of `binding`, with raw pointers on the current stream, against the torch front."""
    import torch
    from paper_2308_07641_b200 import KV4Cache, binding, rotary_table
    g = _gen(5)
    F32, BF16, stream = binding.TSVD_F32, binding.TSVD_BF16, torch.cuda.current_stream().cuda_stream
    # adapters
    a = Adapters(200, 130, [16, 5])
    x, base = torch.randn(9, 200, generator=g, device="cuda"), torch.randn(9, 130, generator=g, device="cuda")
    slots, start = torch.tensor([1, 0], dtype=torch.int32, device="cuda"), torch.tensor([0, 4, 9], dtype=torch.int32, device="cuda")
    want = a.h(x, base, slots, start)
    h = binding.tsvd_adapters_create(200, 130, 16, 2)
    try:
        for s in range(2):
            A, B = a.A[s].float().contiguous(), a.B[s].float().contiguous()
            binding.tsvd_adapters_set(h, s, A.data_ptr(), 200, B.data_ptr(), A.shape[0], F32, A.shape[0], a.c[s], stream)
        for call in (binding.tsvd_adapters_forward, lambda *p: binding.tsvd_adapters_forward_ex(*p[:-1], 0, p[-1])):
            out = torch.zeros_like(want)
            call(h, x.data_ptr(), 200, 0, F32, base.data_ptr(), 130, out.data_ptr(), 130, F32, slots.data_ptr(), start.data_ptr(), 2, 9, stream)
            assert torch.equal(out, want)
        assert binding.tsvd_adapters_info(h)["max_rank"] == 16 and binding.tsvd_adapters_last_status(h) == 0
    finally:
        binding.tsvd_adapters_destroy(h)
    # rotation and the window with first positions
    rates = 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64, device="cuda") / 64)
    table = torch.zeros(300, 64, device="cuda")
    binding.tsvd_rotary_table(table.data_ptr(), 300, 64, rates.data_ptr(), 1.0, stream)
    assert torch.equal(table, rotary_table(300, 64, rates=rates))
    caches = [KV4Cache(2, 64, 20, 16) for _ in range(2)]
    q, k, v = (torch.randn(300, heads, 64, generator=g, device="cuda").bfloat16() for heads in (4, 2, 2))
    pages, n = torch.arange(20, dtype=torch.int32, device="cuda").view(1, 20), torch.tensor([300], dtype=torch.int32, device="cuda")
    first = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
    turned = caches[0].append_rotated(q, k, v, table, pages, n, first)
    want = caches[0].attend(turned, pages, n, first, max_q=300, window=70, sinks=5)
    turned2, out = torch.zeros_like(turned), torch.zeros_like(want)
    batch = (pages.data_ptr(), 20, n.data_ptr(), first.data_ptr(), 1, 300)
    binding.tsvd_kv4_append_rotated(caches[1].handle, q.data_ptr(), 256, turned2.data_ptr(), 256, 4, k.data_ptr(), 128, v.data_ptr(), 128, BF16,
                                    table.data_ptr(), 300, 64, 0, *batch, stream)
    binding.tsvd_kv4_attend_sinks(caches[1].handle, turned2.data_ptr(), 256, out.data_ptr(), 256, 4, BF16, *batch, 300, 0, 0.125, 70, 5,
                                  binding.TSVD_FLAG_CAUSAL, stream)
    torch.cuda.synchronize()
    assert torch.equal(turned2, turned) and torch.equal(out, want)
    assert all(c.status() == 0 for c in caches)


def test_beside_other_cluster_kernels_on_two_streams():
    """The first product of whole sequences, whose blocks share SMs, on one stream; on the other the ternary kernel for 5 to 32 tokens and
    the 8-bit product of few tokens, whose clusters hold tensor memory while they wait for one another.  Same bits as one by one."""
    import torch
    from paper_2308_07641_b200 import Int8Linear, TSVDLinear, quantize
    g, rng = _gen(31), np.random.default_rng(31)
    N = 2048
    ternary = TSVDLinear(rng.integers(-1, 2, (4096, 1024), dtype=np.int8), rng.random(1024, dtype=np.float32) / 64, rng.integers(-1, 2, (1024, N), dtype=np.int8))
    dense = Int8Linear(*quantize(torch.randn(2304, N, generator=g, device="cuda")))
    a = Adapters(N, 640, [128, 20, 64])
    new, slots = [130, 300, 70, 200], [0, 1, -1, 2]
    x = torch.randn(sum(new), N, generator=g, device="cuda").bfloat16()
    base = torch.randn(sum(new), 640, generator=g, device="cuda").bfloat16()
    ids, start, few = torch.tensor(slots, dtype=torch.int32, device="cuda"), _start(new), x[:16].clone()
    ternary.reserve(16, "bf16")
    dense.reserve(16, "bf16")
    want_a = a.check(x, base, slots, new)
    want_t, want_d = ternary(few), dense(few)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [[], []]
        for _ in range(10):
            with torch.cuda.stream(streams[0]):
                got[0].append(a.h(x, base, ids, start))
            with torch.cuda.stream(streams[1]):
                got[1] += [(ternary(few), dense(few))]
        torch.cuda.synchronize()
        assert all(torch.equal(y, want_a) for y in got[0])
        assert all(torch.equal(t, want_t) and torch.equal(d, want_d) for t, d in got[1])
    assert a.h.status() == 0 and dense.status() == 0
