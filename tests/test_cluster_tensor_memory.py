"""Every cluster kernel that uses tensor memory, read off the sources: how its blocks keep from waiting for each other's columns."""
import glob
import os
import re

from tests.test_tensor_memory_order import CSRC, _kernels

CLUSTER_WAITS = r"cluster_sync_all\(\)|barrier\.cluster\.wait"


def test_no_block_waits_for_its_cluster_with_columns_that_another_block_may_want():
    """A block that waits for its cluster while it holds tensor memory must not share an SM with another such block: each could hold
    the columns that a peer of the other's still has to get, and an allocation has no time limit.  So either the launches of such a
    kernel ask for more than half of an SM's shared memory, or every block gives its columns back before it first waits for the
    others."""
    alone, early = set(), set()
    for path, _, body in _kernels():
        waits = [m.start() for m in re.finditer(CLUSTER_WAITS, body)]
        if "tmem_alloc(" not in body or not waits:
            continue
        if body.rindex("tmem_dealloc(") < min(waits):
            early.add(path)
            # what the columns held has been read by then, by all warps: the last loads, a fence, a meeting, a fence, and only then
            tail = body[body.rindex("tmem_ld_wait()"):min(waits)]
            order = [tail.index(s) for s in ("tc_fence_before_sync()", "__syncthreads()", "tc_fence_after_sync()", "tmem_dealloc(")]
            assert order == sorted(order), path
        else:
            alone.add(path)
            text = open(os.path.join(CSRC, path)).read()
            assert re.search(r"std::max(<size_t>)?\([^;]*TSVD_ALONE_SMEM\)", text), \
                f"{path}: a kernel waits for its cluster with columns, and may share an SM"
    assert "adapters.cu" in early and {"i8_mma.cu", "midbatch.cu"} <= alone
    # no file's kernels go unseen
    holders = {os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.cu")) if "tmem_alloc(" in open(p).read()}
    assert holders == {path for path, _, body in _kernels() if "tmem_alloc(" in body}
