"""Scratch of the one kind of drafted-tree kernel that has any: four row blocks over quantised pages, whose registers do not hold all of a walk."""
import re

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


def test_scratch_stays_small(kernels):  # noqa: F811
    found = {name: k for name, k in kernels.items() if re.search(r"draft_tree_kernelINS_\d+B?F16ELi[48]ELi4E", name)}
    assert len(found) == 4
    for name, k in found.items():
        assert k[".vgpr_spill_count"] <= 32 and k[".private_segment_fixed_size"] <= 112, name
