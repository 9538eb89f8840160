"""Scratch memory of the kernels of a cache in 4 bits, from the metadata of the code objects in libfbq.so.  Loads from it wait for what else is under way.  None have any but the many-row kernels (a launch of
their own, or beside the rows' own tokens) of heads of 128 and 256 features, whose two kinds of work - operands made for the next step, products of this one - do not fit a wave's registers: there it
is held to what it was when they were timed."""
import re

from test_kernel_resources import code_objects, kernels  # noqa: F401

BYTES = {("many", "F16", 4): 36, ("many", "Bf16", 4): 96, ("many", "F16", 8): 156, ("many", "Bf16", 8): 724, ("both", "F16", 4): 28, ("both", "Bf16", 4): 84}


def test_scratch_memory(kernels):  # noqa: F811
    found = {n: k for n, k in kernels.items() if re.search(r"fbq_(attend4_\w+|weigh_\w+|append4|evict_\w+|cache_read)_kernel", n)}
    assert len(found) == 10 + 10 + 6 + 40 + 20 + 4 + 5
    for n, k in found.items():
        of = re.search(r"attend4_(many|both)_kernel<(?:fbq::)?Type(\w+), .*?(\d)>", n)
        most = BYTES.get((of[1], of[2], int(of[3])), 0) if of else 0
        assert k[".private_segment_fixed_size"] <= most, (n, k[".private_segment_fixed_size"])
        if not most:
            assert k[".vgpr_spill_count"] == 0, n
