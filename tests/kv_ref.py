"""The cache operators in 64 bits, and how far a result of one rounding may be off."""
import math

import torch

from paper_2608_24658_gb300.api import Rotary

PAGE = 16
ROWS = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.bfloat16}
POOL = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
# half a step, relative to the value
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24, torch.float8_e4m3fn: 2.0 ** -4}
# half of the smallest step (subnormals)
TINY = {torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150, torch.float8_e4m3fn: 2.0 ** -10}


def rows(gen, tokens, heads, d, dtype, pad=0, heads_first=False):
    """[tokens, heads, d] of N(0, 1), as a view with `pad` elements between tokens."""
    if heads_first:
        x = torch.randn((heads, tokens, d + pad), generator=gen, device="cuda").to(dtype)
        return x[..., :d].transpose(0, 1)
    x = torch.randn((tokens, heads * d + pad), generator=gen, device="cuda").to(dtype)
    return x[:, pad:].unflatten(1, (heads, d))


def rotary_of(kind):
    """(Rotary or None, axis of each frequency) of a short description."""
    if kind is None:
        return None, None
    dim, axes, interleaved = kind
    half = dim // 2
    inv = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()
    table = [i % axes for i in range(half)] if axes > 1 else None
    return Rotary(inv, axes=table, interleaved=interleaved), table or [0] * half


def rotated(x, rotary, table, positions):
    """(x rotated in 64 bits, |p| + |q| of each element's pair)."""
    y = x.double().clone()
    size = torch.zeros_like(y)
    if rotary is None:
        return y, size
    pos = positions.reshape(-1, x.shape[0]).double()
    freq = rotary.inv_freq.double()
    angle = torch.stack([pos[a] * freq[i] for i, a in enumerate(table)], dim=1).unsqueeze(1)
    c, s = torch.cos(angle), torch.sin(angle)
    half = len(table)
    lo, hi = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if rotary.interleaved
              else (slice(0, half), slice(half, 2 * half)))
    p, q = x[..., lo].double(), x[..., hi].double()
    y[..., lo], y[..., hi] = p * c - q * s, p * s + q * c
    size[..., lo] = size[..., hi] = p.abs() + q.abs()
    return y, size


def bound(ref, size, dtype, steps=1):
    """One rounding to `dtype` of a value that fp32 arithmetic has off by a few
    2^-24 of what went into it: cos and sin are off by at most 2^-22 (half a turn's
    fraction rounds to 2^-26 of a turn, times 2 pi, and two units of sincospi),
    a product and a sum round twice, a division or product with a scale `steps`
    times more."""
    off = 2.0 ** -21 * size + steps * 2.0 ** -24 * ref.abs()
    return off + HALF[dtype] * (ref.abs() + off) + TINY[dtype]


def stored(ref, size, scale):
    """What the e4m3 cache is to hold: the quotient, saturated, and its pair's size."""
    s = scale.double().view(-1, 1)
    return (ref / s).clamp(-448.0, 448.0), size / s


def raw(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def pool(gen, pages, heads, d, mode):
    """Pools whose slots hold random bits (NaN among them)."""
    n = torch.empty(0, dtype=POOL[mode]).element_size()
    return [torch.randint(0, 256, (pages, heads, PAGE, d * n), generator=gen, device="cuda",
                          dtype=torch.uint8).view(POOL[mode]) for _ in range(2)]


def at(pages, slots):
    """Rows [T, heads, d] of the slots, raw."""
    s = slots.long()
    return raw(pages)[s // PAGE, :, s % PAGE]


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen
