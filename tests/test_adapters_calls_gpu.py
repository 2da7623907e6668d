"""The adapters where a call meets its surroundings: waits that give up.  (Tolerances: test_norm_adapters_gpu.)"""
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
