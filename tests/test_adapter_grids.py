"""How many blocks of the adapters' second kernel are taken to run at a time, read off the source."""
import os
import re

from tests.test_layer_front import _body
from tests.test_tensor_memory_order import CSRC


def test_the_second_kernel_counts_the_blocks_that_an_sm_holds():
    """Its grid is sized for one round: from the registers that its launch bounds leave and from its shared memory, not from a number for
    all types and ranks."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "adapters.cu")).read())
    start = text.index("cudaError_t up(UpParams& p")
    rule = text[start:text.index("cudaLaunchKernelEx(", start)]
    assert re.search(r"fit = \(int\)\(TSVD_SM_SMEM / \(smem \+ kUpStatic\)\)", rule)
    assert re.search(r"at_once = sms \* std::max\(1, std::min\(\{fit, kUpBlocks<T, G>, most\}\)\)", rule)
    assert re.search(r"tiles \* columns\(\) > at_once", rule) and re.search(r"l\(\(unsigned\)tiles, UP_WARPS \* 32, smem, st\)", rule)
    # what the kernel declares, and the kilobyte that the system keeps
    rows = int(re.search(r"UP_ROWS = (\d+);", text).group(1))
    declared = 0
    for line in re.findall(r"__shared__ (?:int|unsigned) ([^;]+);", _body("adapters.cu", "adapter_up_kernel")):
        for size in re.findall(r"\w+(?:\[([^\]]+)\])?(?:,|$)", line):
            declared += 4 * (eval(size, {"UP_ROWS": rows}) if size else 1)
    assert 1024 < declared + 1024 <= int(re.search(r"kUpStatic = (\d+);", text).group(1))
