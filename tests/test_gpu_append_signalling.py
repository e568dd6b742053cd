"""Signalling not-a-numbers of rows on their way into pages take no part in a row's range or in statistics, like any other."""
import numpy as np
import pytest
import torch

from test_gpu_append_special import SIGNALLING, _append, _expected
from test_gpu_quant import _unpack_rows

pytestmark = pytest.mark.gpu


def _numbers(x):
    """In 32 bits, every not-a-number a quiet one: numpy's own reductions would take a signalling one for what came before it."""
    f = x.float().numpy()
    return np.where(np.isnan(f), np.float32(np.nan), f)


@pytest.mark.parametrize("one_by_one", [False, True])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("seed", [8, 9, 10])
def test_extremes_next_to_signalling_not_a_numbers(dtype, bits, one_by_one, seed):
    """The extremes of a row in front of one, behind one and between two, at every place of the eight channels that a lane has."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((40, 128), generator=g).to(torch.float16 if dtype == "fp16" else torch.bfloat16)
    raw = x.view(torch.int16)
    for i in range(32):  # lane i / 2's channels: the row's extremes at two of them, not-a-numbers at the others, or at half of the others
        first = 8 * (i // 2)
        for c in range(first, first + 8):
            if i % 2 or c % 2:
                raw[i, c] = SIGNALLING[dtype] - (0x8000 if c % 3 else 0)
        low, high = first + (seed + i) % 8, first + (seed + 3 * i + 5) % 8
        x[i, low] = -40.0
        x[i, high if high != low else first + (low + 1) % 8] = 50.0
    raw[39] = SIGNALLING[dtype]  # nothing but
    k, v, stats = _append(x, bits, dtype, one_by_one)
    codes, scale, zero = _expected(_numbers(x), bits)
    size = 64 * 128 * bits // 8
    for pool in (k, v):
        slab = pool.numpy()[0, 0]
        pair = np.ascontiguousarray(slab[size:]).view(np.float16).reshape(64, 2)[:40]
        assert np.array_equal(pair[:, 0], scale, equal_nan=True) and np.array_equal(pair[:, 1], zero, equal_nan=True)
        assert np.array_equal(_unpack_rows(slab[:size].reshape(64, 128 * bits // 8), bits)[:40], codes)
    for page in range(3):
        part = _numbers(x)[16 * page:16 * page + 16]
        high, low = np.fmax(np.fmax.reduce(part, axis=0), -np.inf), np.fmin(np.fmin.reduce(part, axis=0), np.inf)
        assert np.array_equal(stats[0, 0, page, 0].float().numpy(), high) and np.array_equal(stats[0, 0, page, 1].float().numpy(), low)
