"""Values of quantised pages of a bf16 layer, whose range fp16 does not have: tiny rows and loud ones."""
import numpy as np
import pytest
import torch

from test_gpu_tree_pages import _set_row
from tree_reference import Problem

pytestmark = pytest.mark.gpu


def _problem(bits, nodes, lens=(300,), **kw):
    """Tokens that attend the history alone, so that nothing of theirs covers what comes out of it."""
    none = [np.zeros((nodes, nodes), dtype=bool)] * len(lens)
    return Problem(lens, [[-1] * nodes] * len(lens), dtype=torch.bfloat16, bits=bits, flags=[0, 0], see=none, **kw)


def _check(p):
    """(values as they are meant: rounding of the weights to 11 bits and of the result to 8, which Problem.check allows for and more)"""
    import paper_2502_14866_amd as L

    L.load_library()
    out, lse = p.call(L)
    p.check(out, lse)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("nodes", [2, 40])
@pytest.mark.parametrize("steps,zero", [(1, 0.0), (3, 0.0), (7, 2.0 ** -23), (33, -2.0 ** -20), (1, 2.0 ** -24)])
def test_tiny_rows(bits, nodes, steps, zero):
    """Scales of a few steps of fp16's smallest numbers."""
    p = _problem(bits, nodes)
    for hk in range(2):
        for t in range(300):
            _set_row(p, "v", 0, hk, t, steps * 2.0 ** -24, zero)
    _check(p)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("nodes", [2, 40])
def test_loud_rows(bits, nodes):
    """Values up to some millions, from scales and zeros that fp16 has, beside ordinary ones."""
    p = _problem(bits, nodes, (300, 128))
    for b, hk in ((0, 0), (0, 1), (1, 1)):
        for t in range(0, p.lens[b], 2):
            _set_row(p, "v", b, hk, t, 8000.0, (-60000.0, 65504.0)[t // 2 % 2])
    _check(p)
