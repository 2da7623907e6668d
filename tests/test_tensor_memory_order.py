"""What keeps kernels from waiting for each other's tensor memory, read off the sources: an allocation has no time limit, so that it
ends is a matter of construction and not of a run."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2308_07641_b200", "csrc")


def _kernels():
    """(file, name, body) of every __global__ function."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__[^{;]*?(\w+)\s*\(([^{;]*)\)\s*\{", text):
            depth, i = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[i], 0)
                i += 1
            yield os.path.basename(path), m.group(1), text[m.end():i]


def test_tensor_memory_is_allocated_before_the_next_kernel_may_start():
    """Else a later kernel of the stream can hold the columns, waiting for one that still has to get them."""
    seen = set()
    for path, name, body in _kernels():
        if "tmem_alloc(" not in body:
            continue
        seen.add(path)
        assert body.count("tmem_alloc(") == 1, name
        for call in ("pdl_launch_dependents()", "pdl_wait()"):
            first = body.find(call)
            assert first < 0 or body.index("tmem_alloc(") < first, f"{path}: {name} calls {call} before it has its tensor memory"
        # every way out gives it back
        assert body.count("tmem_dealloc(") == 1 + len(re.findall(r"\breturn\s*;", body[body.index("tmem_alloc("):])), f"{path}: {name}"
    assert {"kv4_prefill.cu", "i8_mma.cu", "midbatch.cu", "tensor.cu"} <= seen


@pytest.mark.parametrize("path", ["i8_mma.cu", "midbatch.cu"])
def test_cluster_kernels_with_tensor_memory_have_an_sm_to_themselves(path):
    """Their blocks wait for one another while they hold columns: two on an SM, of different clusters, could each wait for what
    the other one holds.  More than half of an SM's shared memory keeps them apart (a static_assert says that it is)."""
    both = [name for p, name, body in _kernels() if p == path and "tmem_alloc(" in body and "cluster_sync_all()" in body]
    assert both
    text = open(os.path.join(CSRC, path)).read()
    assert re.search(r"std::max(<size_t>)?\([^;]*TSVD_ALONE_SMEM\)", text), "the launch does not ask for the shared memory"
    head = open(os.path.join(CSRC, "tsvd_internal.cuh")).read()
    alone, sm = (eval(re.search(r"constexpr size_t " + n + r" = ([\d *]+);", head).group(1)) for n in ("TSVD_ALONE_SMEM", "TSVD_SM_SMEM"))
    assert 2 * alone > sm == 228 * 1024


def test_dependents_do_not_promise_that_their_inputs_stay():
    """A kernel that starts before the one ahead of it has ended must not read that one's results as data that never change
    (__ldg, const __restrict__): such loads may move ahead of its wait.  The serving kernels have none."""
    seen = set()
    for path in ("quant8.cu", "rows8.cuh", "i8_mma.cu", "kv4.cu", "kv4_decode.cu", "kv4_prefill.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
        assert "__ldg(" not in text and "ld.global.nc" not in text, path
        for m in re.finditer(r"__global__[^{;]*?(\w+)\s*\(([^{;]*)\)\s*\{", text):
            if "pdl_wait()" in text[m.end():m.end() + 4000]:
                seen.add(path)
                assert not re.search(r"const\s+[\w<>]+\s*\*\s*__restrict__", m.group(2)), f"{path}: {m.group(1)}"
    assert len(seen) == 6


def test_ternary_dependents_do_not_promise_it_either():
    """The same for the ternary kernels: read-only loads only of what belongs to the handle and no kernel writes."""
    for path in ("digits.cuh", "tensor.cu", "decode.cu", "index.cu", "midbatch.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
        for m in re.finditer(r"__ldg\(([^)]*)\)", text):
            assert re.match(r"p\.(bias|row_ptr|entries)\b", m.group(1)), f"{path}: {m.group(0)}"
        for m in re.finditer(r"const\s+(\w+)\s*\*\s*__restrict__\s+(\w+)", text):
            raise AssertionError(f"{path}: {m.group(0)}")
