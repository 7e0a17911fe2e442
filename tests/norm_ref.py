"""The norm of each head in 64 bits, with the rotation behind it, and how far fp32 is off."""
import torch

from tests import kv_ref as R

EPS = 1e-6


def weight(gen, shape, dtype, offset=0.0):
    return (1.0 - offset + 0.3 * torch.randn(shape, generator=gen, device="cuda")).to(dtype)


def rows(x, w, rotary, table, positions, eps=EPS, offset=0.0):
    """x [T, H, d] normed by w ([d] or [H, d]; None: not) and rotated, and its pairs' |p| + |q|."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt(y.square().mean(dim=-1, keepdim=True) + eps) * (w.double() + offset)
    return R.rotated(y, rotary, table, positions)


def loose(ref, size):
    """Before any rounding to fewer bits.  A norm: each square rounds once, and their sum 16
    + 7 times (2^-24 each, relative, all squares being positive), the mean with eps and its
    reciprocal root twice, of which a root keeps half; three products or sums with the weight: below
    18 units of 2^-24, for each element of a pair.  A rotation: 2^-21 of the pair (kv_ref)."""
    return (2.0 ** -21 + 18 * 2.0 ** -24) * size + 18 * 2.0 ** -24 * ref.abs() + 2.0 ** -120
