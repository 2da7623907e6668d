"""Norms of finite rows whose products with the weights leave fp32's range."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2308_07641_b200 import build
    build.build()


@pytest.mark.parametrize("cols", [40, 300, 4096, 40000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_products_beyond_fp32(cols, dtype):
    """As numbers the row is scaled before the weights come in, and stays what it is (tolerance of test_norm_adapters_gpu: (n / 64 + 18) u and
    the result's rounding); in 8 bits its scale says that it cannot be had.  The rows beside it know nothing of it."""
    import torch
    from paper_2308_07641_b200 import rms_norm, rms_norm_quantize
    kind = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    x = torch.randn(6, cols, generator=g, device="cuda")
    x[1] *= 1e30
    x[4, cols // 2] = 3e38
    x, w = x.to(kind), 1e9 * (1 + torch.rand(cols, generator=g, device="cuda"))
    d = x.double()
    want = d / (d.square().mean(1, keepdim=True) + 1e-6).sqrt() * w.double()
    tol = ((cols / 64 + 18) * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)) * want.abs() + 1e-30
    assert ((rms_norm(x, w).double() - want).abs() <= tol).all()
    q, scale = rms_norm_quantize(x, w)
    assert torch.isinf(scale[[1, 4]]).all() and torch.isfinite(scale[[0, 2, 3, 5]]).all()
    fine = [0, 2, 3, 5]
    q2, scale2 = rms_norm_quantize(x[fine], w)
    assert torch.equal(q[fine], q2) and torch.equal(scale[fine], scale2)
