"""What makes a wait that gave up end its kernel, read off the sources of the attention over the 4-bit cache."""
import re

import pytest

from tests.test_tensor_memory_order import _kernels


@pytest.mark.parametrize("path", ["kv4_decode.cu", "kv4_prefill.cu"])
def test_a_warp_agrees_on_a_wait_that_gives_up(path):
    """Where a phase ends as the limit does, the lanes of a warp may see different answers; those that go on would wait for the
    others for ever.  So a warp waits with mbar_wait_warp, and with mbar_wait only one elected lane, or lanes that compare their
    answers (`ok`) before any leaves."""
    found = 0
    for p, name, body in _kernels():
        if p != path:
            continue
        elected = []                                         # what lies inside `if (elect_one() ...) { ... }`
        for m in re.finditer(r"if \(elect_one\(\)[^{]*\{", body):
            depth, i = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(body[i], 0)
                i += 1
            elected.append((m.end(), i))
        for m in re.finditer(r"\bmbar_wait\(", body):
            if any(a < m.start() < b for a, b in elected):
                continue
            rest = body[body.rindex("\n", 0, m.start()):]
            assert rest.lstrip().startswith("ok = mbar_wait("), f"{name}: {rest[:60]}"
            assert "break" not in rest[:rest.index("__all_sync(0xffffffffu, ok)")], name
        found += len(re.findall(r"\bmbar_wait_warp\(", body))
    assert found
