"""Orders in the kernels' sources that no run shows until it hangs."""
import os
import re

import pytest

import paper_2609_32398_gb300

CSRC = os.path.join(os.path.dirname(paper_2609_32398_gb300.__file__), "csrc")


@pytest.mark.parametrize("name", ["experts_product.cu", "experts_wgrad.cu"])
def test_tensor_memory_is_taken_after_the_kernel_before(name):
    """A programmatic dependent may share its SM with the kernel before: if it took all of
    the tensor memory and then waited for that kernel, one that has still to take its own would
    wait for it in turn."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    waits = [m.start() for m in re.finditer(r"\bpdl_wait\(\)", code)]
    takes = [m.start() for m in re.finditer(r"\bpair_tmem_alloc\(", code)]
    assert len(waits) == 1 and len(takes) == 1 and waits[0] < takes[0]
