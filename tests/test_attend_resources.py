"""Registers, scratch memory and LDS of the attention kernels, from the metadata of the code objects in libfbq.so: their launch shapes count on a number of blocks a CU, and a
load from scratch memory in a loop waits for every copy that is under way (heads of 256 took eight times as long with it)."""
import re

from test_kernel_resources import code_objects, kernels  # noqa: F401


def test_attention_kernels_have_their_registers_and_no_scratch(kernels):  # noqa: F811
    found = {n: k for n, k in kernels.items() if re.search(r"fbq_(attend|join)_\w+_kernel<", n)}
    assert len([n for n in found if "fbq_attend_few_kernel<" in n]) == 6          # 2 types x (64, 128, 256 features)
    assert len([n for n in found if "fbq_attend_many_kernel<" in n]) == 8         # 2 types x (64, 96, 128, 256)
    assert len([n for n in found if "fbq_attend_both_kernel<" in n]) == 6         # 2 types x (64, 96, 128)
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n
        if "join" in n:
            continue
        alone = "256" in n                                                       # one block a CU, else two
        assert k[".vgpr_count"] <= (512 if alone else 256), (n, k[".vgpr_count"])   # (accumulation registers among them)
        assert k[".group_segment_fixed_size"] <= (160 if alone else 80) * 1024, n
