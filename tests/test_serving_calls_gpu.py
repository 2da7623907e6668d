"""The serving operators where a call meets its surroundings: devices, streams, launches in a chain, rows of unlike size."""
import ctypes

import pytest

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
