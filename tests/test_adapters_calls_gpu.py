"""The adapters where a call meets its surroundings: waits that give up, results that are exact.  (Tolerances: test_norm_adapters_gpu.)"""
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
