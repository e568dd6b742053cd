"""What the kernels of drafted trees and of new tokens occupy, from the metadata of the built library."""
import re

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


def test_two_workgroups_of_drafted_trees_fit_a_compute_unit(kernels):  # noqa: F811
    """64 KiB of tiles each, and two wavefronts to a SIMD where a workgroup has four."""
    seen = 0
    for name, k in kernels.items():
        m = re.search(r"draft_tree_kernelINS_\d+B?F16ELi(\d+)ELi(\d+)E", name)
        if not m:
            continue
        bits, blocks = map(int, m.groups())
        seen += 1
        assert k[".group_segment_fixed_size"] <= 80 * 1024, name
        assert k[".vgpr_count"] <= 256, name
        if bits == 16 or blocks == 2:
            assert k[".private_segment_fixed_size"] == 0, name
    assert seen == 2 * (3 + 2 + 2)  # types; blocks of 32 rows to a workgroup over pages of 16, 8 and 4 bits


def test_the_others_use_no_scratch(kernels):  # noqa: F811
    found = [k for name, k in kernels.items()
             if re.search(r"fold_trees_kernel|extend_tables_kernel|tree_masks_kernel|rotary_rows_kernel|rotary_pairs_kernel", name)]
    assert len(found) == 2 * 3 + 1 + 3 + 2 * 2 + 2 * 2
    assert all(k[".private_segment_fixed_size"] == 0 for k in found)
