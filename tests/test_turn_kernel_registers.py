"""What the kernels that turn rows occupy, from the metadata of the built library."""
import re

from test_kernel_registers import kernels  # noqa: F401  (the fixture)


def _found(kernels, pattern):  # noqa: F811
    return {name: k for name, k in kernels.items() if re.search(pattern, name)}


def test_no_scratch(kernels):  # noqa: F811
    found = _found(kernels, r"turned_(rows|pairs|append|step)_kernel")
    assert len(found) == 2 * (3 * 2 + 2 + 2 * 3 * 3 * 2)  # types; layouts and norms of rows, layouts of pairs; layouts, bits and norms of the other two
    assert all(k[".private_segment_fixed_size"] == 0 for k in found.values())


def test_wavefronts_to_a_unit(kernels):  # noqa: F811
    """Rows in flight are what these kernels need: five wavefronts to a SIMD for rows (102 registers) and three into pages (168), five of those without a
    norm into 16-bit pages where no row passes through LDS."""
    for k in _found(kernels, r"turned_rows_kernel").values():
        assert k[".vgpr_count"] <= 102
    for name, k in _found(kernels, r"turned_append_kernel").items():
        assert k[".vgpr_count"] <= 168
        if re.search(r"ELi[01]ELi16ELb0E", name):
            assert k[".vgpr_count"] <= 102, name
