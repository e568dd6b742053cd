"""The cases of perf/more_operators.py, listed ones and drawn ones, by the library and in plain form against their definition in 64 bits."""
import importlib.util
import os
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("more_operators", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "more_operators.py"))
M = importlib.util.module_from_spec(spec)
spec.loader.exec_module(M)

MOST = 2e8  # bytes that a drawn case moves


def _drawn(n):
    rng, out = random.Random(12), []
    while len(out) < n:
        case = M.draw(rng)
        if M.work(case)["bytes"] <= MOST:
            out.append(case)
    return out


CASES = M.listed() + _drawn(24)


def _made(case, own):
    M.own = own
    try:
        out = M.run(M.prepare(case, 7))
        torch.cuda.synchronize()
        return out
    finally:
        M.own = False


def _tolerance(case, name, want, sums):
    """Half a step of the type, and what 32-bit arithmetic is off by before: with M the largest output, a pair is 2 sqrt(2) M at most in sum of sizes; angle, sine, cosine,
    products and sum are 4.6e-7 of it, a norm 14 U, taking off the mean another 12 U, in all below 8e-6 M (`sums`: a row's sum added in another order, 127 U of it at most
    instead of 19).  What is kept in codes is off by these, then by a whole code where a rounding went the other way, and, as scale and zero are rounded to fp16 and the value
    to the layer's type, by 2^-10 of the row's range and ends and a step of the type."""
    t = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
    half = torch.finfo(t).eps / 2
    near = half * want.abs() + half * torch.finfo(t).smallest_normal + sums * want.abs().max()
    if case.get("kv_bits", 16) == 16 or name not in ("k_pool", "v_pool", "k_stream", "v_stream"):
        return near
    high, low = want.amax(-1, keepdim=True), want.amin(-1, keepdim=True)
    return near + half * want.abs() + (high - low) / (2 ** case["kv_bits"] - 1) + (high - low + high.abs().maximum(low.abs())) * 2.0 ** -10 + 2 * half * high.abs().maximum(low.abs())


@pytest.mark.parametrize("case", CASES, ids=[c.get("name", f"drawn_{i}") for i, c in enumerate(CASES)])
def test_against_the_definition(case):
    want = M.exact(case, 7)
    for own in (True, False):
        made = _made(case, own)
        assert set(made) == set(want)
        for name, ref in want.items():
            got = made[name].double()
            assert got.shape == ref.shape and ((got - ref).abs() <= _tolerance(case, name, ref, 8e-6 if own else 2e-5)).all(), (name, own, float((got - ref).abs().max()))
