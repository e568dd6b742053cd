"""Heads normed and turned, from the formulas in 64 bits, with how far 32-bit arithmetic may be off before the result is rounded."""
import torch

U = 2.0 ** -24  # half a step of fp32


def reference(x, R, interleaved, positions, pair_axis, freq, scale=1.0, norm=None, weight=None, eps=1e-6):
    """x [n][heads][D] on the CPU, positions [axes][n], norm None, "rms" or "centred".  (result, bound) in 64 bits.

    Norm: the squares are added in a chain of 16 fused steps, three more sums over lanes (19 U of the sum, all terms positive; other kernels take
    fewer), eps one more U; the inverse root has half of that and two U of its own: 12 U; times x and times the weight: 14 U of the result.  Centred: a mean of
    128 values is off by 12 U of the mean magnitude A at most (nine sums of a lane, three over lanes), which moves every channel by as much, times inverse root and
    weight; the difference has a U of its own, 15 U; the sum of squares moves by 128 of these shifts squared.
    Turn: angle, sine, cosine, scale, products and sum 4.6e-7 of |a| + |b| (0.94e-7, 1.2e-7, 2.4e-7), 2^-51 of the angle, and what a and b are off by."""
    y, D = x.double(), x.shape[-1]
    off = torch.zeros_like(y)
    if norm:
        eps = float(torch.tensor(eps, dtype=torch.float32))
        size = y.abs().mean(-1, keepdim=True)
        if norm == "centred":
            y = y - y.mean(-1, keepdim=True)
        var = (y * y).mean(-1, keepdim=True) + eps
        w = torch.ones(D, dtype=torch.float64) if weight is None else weight.double()
        y = y / var.sqrt() * w
        off = 14 * U * y.abs()
        if norm == "centred":
            shift = 12 * U * size
            off = (15 * U + shift ** 2 / (2 * var)) * y.abs() + shift / var.sqrt() * w.abs()
    out, bound = y.clone(), off.clone()
    if R:
        ia = torch.arange(0, R, 2) if interleaved else torch.arange(R // 2)
        ib = ia + (1 if interleaved else R // 2)
        angle = positions.double()[torch.as_tensor(pair_axis)[:R // 2]].t() * freq
        c, s = angle.cos()[:, None], angle.sin()[:, None]
        a, b = y[..., ia], y[..., ib]
        out[..., ia], out[..., ib] = scale * (a * c - b * s), scale * (b * c + a * s)
        both = scale * (off[..., ia] + off[..., ib] + (a.abs() + b.abs()) * (4.6e-7 + angle.abs()[:, None] * 2.0 ** -51))
        bound[..., ia], bound[..., ib] = both, both
    return out, bound


def assert_close(got, want, dtype):
    """One rounding to the type on top: half a step, or half the smallest number."""
    ref, bound = want
    half = torch.finfo(dtype).eps / 2
    tol = ref.abs() * half + torch.finfo(dtype).smallest_normal * half + bound * (1 + half)
    worst = ((got.cpu().double() - ref).abs() - tol).max()
    assert worst <= 0, float(worst)
