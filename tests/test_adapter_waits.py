"""What the adapters' kernels on tcgen05 leave behind when a wait of theirs gives up, read off the source."""
import re

from tests.test_layer_front import _body


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
