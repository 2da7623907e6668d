"""What the adapters' kernels on tcgen05 leave behind when a wait of theirs gives up, read off the source, and the flag by which a test
makes them."""
import ctypes
import re

import pytest

from tests.test_layer_front import _adapters, _body, front  # noqa: F401
from tests.test_serving_front import OnCard, _status

torch = pytest.importorskip("torch")


def test_weights_on_their_way_land_whoever_gave_up():
    """The first product keeps its parts where the weights were: a copy that still lands, of a wait that the copying warp or the one that
    issues products gave up, has to be waited for after both are done and before the first part is written."""
    body = _body("adapters.cu", "adapter_down_many_kernel")
    parts = body.index("tmem_ld8(")
    met = body.rindex("__syncthreads();", 0, body.index("if (ctl[0])"))            # all warps have ended their loops
    assert body.rindex("mbar_wait(") < met < parts
    drain = re.search(r"if \(ctl\[0\]\) \{\s*if \(threadIdx\.x == 0\)\s*for \(int i = max\(0, asked - STAGES\); i < asked; \+\+i\) "
                      r"mbar_drain\(&w_full\[i % STAGES\], [^;]*\);\s*__syncthreads\(\);\s*\}", body)
    assert drain and met < drain.start() and drain.end() < parts
    assert body.count("mbar_drain(&w_full") == 1


def test_both_kernels_withhold_the_weights():
    """With the test's flag neither kernel asks for a copy of weights, so that nothing is under way when their waits run out, and the limit
    is the short one."""
    for name in ("adapter_down_many_kernel", "adapter_many_kernel"):
        body = _body("adapters.cu", name)
        assert "ctl[1] = p.test_stall ? kWaitLimitStall : kWaitLimitDefault;" in body
        assert body.count("bulk_g2s(") == 1
        guard = body.rindex("if (", 0, body.index("mbar_arrive_expect_tx("))
        assert "!p.test_stall" in body[guard:body.index("{", guard)]


def test_flags(front):  # noqa: F811
    """No other flag than the test's; refused like the sibling calls' are, in C and in the front."""
    binding, serving = front
    a = _adapters(serving)
    card = lambda *s, dtype=torch.float32: OnCard(torch.zeros(*s, dtype=dtype))  # noqa: E731
    x, base, slots = card(5, 8), card(5, 6), card(5, dtype=torch.int32)
    for flags in (binding.TSVD_FLAG_OUT_BF16, binding.TSVD_FLAG_CAUSAL, binding.TSVD_FLAG_TEST_STALL | 1, 1 << 31):
        assert _status(binding, a, x=x, base=base, slots=slots, flags=flags) == binding.TSVD_E_DTYPE
    p = ctypes.c_void_p(64)
    assert binding.lib().tsvd_adapters_forward_ex(None, p, 4, None, 0, p, 4, p, 4, 0, p, None, 1, 1, 0, None) == binding.TSVD_E_NULL
