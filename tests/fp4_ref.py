"""Pools in 4 bits, what they stand for, and attention over them in 64 bits."""
import math
from dataclasses import replace

import numpy as np
import torch

from paper_2608_24658_gb300 import workloads as W

PAGE, BLOCK, D = 16, 16, 128
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
VALUES = torch.cat([VALUES, -VALUES])
NAN_SCALE = 0x7F


def split(pages, d=D):
    """(values [P, H, 16, d / 2], scales [P, H, 16, d / 16]), views of pools of bytes."""
    return (pages[..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2)),
            pages[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // BLOCK)))


def decoded(pages, scale, d=D):
    """[P, H, 16, d] in 64 bits."""
    v, s = split(pages, d)
    table = VALUES.to(pages.device)
    x = table[torch.stack([v & 15, v >> 4], dim=-1).flatten(-2).long()]
    s = s.contiguous().view(torch.float8_e4m3fn).float().double()
    return (x.unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2) * scale.double().view(1, -1, 1, 1)


def random_pool(gen, pages, heads, lo=0x28, hi=0x40, d=D):
    """Bytes of random values; scales from e4m3 codes lo .. hi (0.25 to 2)."""
    pool = torch.randint(0, 256, (pages, heads, 9 * d), generator=gen, device="cuda", dtype=torch.uint8)
    split(pool, d)[1].random_(lo, hi + 1, generator=gen)
    return pool


def tree_of(parent, lens, leaves, h_q, h_kv, seed, prefill=False, q_std=1.0, permute=True, sm_scale=0.0,
            extra_pages=3):
    """A ForkTree in mode fp4; slots that no token holds, and free pages, are NaN."""
    t = W.build_tree("fp4", parent, lens, leaves, num_q_heads=h_q, num_kv_heads=h_kv, head_dim=D, mode="fp4",
                     seed=seed, permute_pages=permute, extra_pages=extra_pages, values=False, sm_scale=sm_scale)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rows = int(sum(lens[n] for n in leaves)) if prefill else len(leaves)
    q = (q_std * torch.randn((rows, h_q, D), generator=gen, device="cuda")).to(torch.bfloat16)
    pools = [random_pool(gen, max(1, t.num_physical_pages), h_kv) for _ in range(2)]
    held = torch.zeros((max(1, t.num_physical_pages), PAGE), dtype=torch.bool)
    for n, tokens in enumerate(lens):
        for i in range(tokens):
            held[t.page_ids[t.node_page_ptr[n] + i // PAGE], i % PAGE] = True
    page, at = (~held).nonzero().T.cuda()
    for p in pools:
        v, s = split(p)
        v[page, :, at] = 0xFF
        s[page, :, at] = NAN_SCALE
    scales = [0.3 + 0.5 * torch.rand(h_kv, generator=gen, device="cuda") for _ in range(2)]
    return replace(t, q=q, k_pages=pools[0], v_pages=pools[1], k_scale=scales[0], v_scale=scales[1])


def slots_of(t, n):
    i = np.arange(int(t.node_len[n]))
    return torch.from_numpy(t.page_ids[t.node_page_ptr[n] + i // PAGE].astype(np.int64) * PAGE + i % PAGE).cuda()


def attend(t, prefill=False, cap=0.0):
    """out, lse, and what their errors scale with: sum p |v|, the largest scale * sum |q k|, and
    the largest p times sum |v|."""
    g = t.num_q_heads // t.num_kv_heads
    scale = t.sm_scale or 1.0 / math.sqrt(D)
    flat = [decoded(p, s).transpose(1, 2).flatten(0, 1) for p, s in ((t.k_pages, t.k_scale), (t.v_pages, t.v_scale))]
    q = t.q.double()
    out, lse, mean, size, tiny, row = [], [], [], [], [], 0
    for leaf in t.leaf_node:
        path, n = [], int(leaf)
        while n >= 0:
            path.append(n)
            n = int(t.parent[n])
        slots = torch.cat([slots_of(t, n) for n in path[::-1]])
        k, v = (x[slots].repeat_interleave(g, dim=1) for x in flat)            # [keys, H_q, d]
        rows = int(t.node_len[leaf]) if prefill else 1
        for i in range(rows):
            seen = len(slots) - rows + 1 + i if prefill else len(slots)
            s = scale * torch.einsum("hd,khd->hk", q[row], k[:seen])
            mass = scale * torch.einsum("hd,khd->hk", q[row].abs(), k[:seen].abs())
            s = cap * torch.tanh(s / cap) if cap else s
            z = torch.logsumexp(s, dim=-1) if seen else torch.full((t.num_q_heads,), -math.inf, device="cuda",
                                                                   dtype=torch.float64)
            p = torch.exp(s - z.unsqueeze(-1))
            out.append(torch.einsum("hk,khd->hd", p, v[:seen]))
            mean.append(torch.einsum("hk,khd->hd", p, v[:seen].abs()))
            tiny.append(v[:seen].abs().sum(dim=0) * (p.amax(dim=-1, keepdim=True) if seen else 0.0))
            size.append(mass.amax(dim=-1) if seen else torch.zeros_like(z))
            lse.append(z)
            row += 1
    return tuple(torch.stack(x) for x in (out, lse, mean, size, tiny))


def check(t, out, lse, prefill=False, cap=0.0):
    """Scores: products of f16 numbers are exact, their sums of 128 lose at most 128 units of 2^-23 of
    the sum of magnitudes, the cap (a series or exponentials in fp32) 2^-19 of itself.  P: an error
    of a score is one of its exponential, which rounds to f16 (2^-11; a subnormal, below 2^-14
    of the largest, by 2^-25 of it: every piece of the keys has a P of 1 or more) after 2^-21 of ex2, and
    the sums of P V lose as much again as the scores; partial results join in fp32 (2^-20).  The
    result rounds to bf16 (2^-8)."""
    ref, z, mean, size, tiny = attend(t, prefill, cap)
    score = 2.0 ** -16 * size + 2.0 ** -19 * cap
    fine = torch.isfinite(z)
    assert torch.equal(torch.isfinite(lse), fine) and torch.equal(lse[~fine].double(), z[~fine])
    off = (lse.double() - z).abs()[fine]
    most = (score + 2.0 ** -20 * (1.0 + z.abs()))[fine]
    assert (off <= most).all(), float((off / most).max())
    p = 2.0 ** -11 + 2.0 ** -15 + 2 * score.unsqueeze(-1)
    off = (out.double() - ref).abs()
    most = 2.0 ** -8 * ref.abs() + (1 + 2.0 ** -8) * (p * mean + 2.0 ** -25 * tiny)
    assert (off <= most).all(), float((off - most).max())
    assert (out[~fine] == 0).all()
