"""Capped attention of a fork tree in 64 bits, and how far the kernels may be off."""
import math

import numpy as np
import torch

# half a step of P and of the result, relative (fp32 mode keeps P in fp32)
P_HALF = {"bf16": 2.0 ** -8, "fp8": 2.0 ** -11, "fp32": 2.0 ** -24}
OUT_HALF = {"bf16": 2.0 ** -8, "fp8": 2.0 ** -8, "fp32": 2.0 ** -24}


def node_kv(tree, n):
    """K and V of node n, [H_kv, tokens, d], in 64 bits."""
    lo, hi = int(tree.node_page_ptr[n]), int(tree.node_page_ptr[n + 1])
    ids = torch.as_tensor(tree.page_ids[lo:hi].astype(np.int64), device=tree.k_pages.device)
    got = []
    for pages, scale in ((tree.k_pages, tree.k_scale), (tree.v_pages, tree.v_scale)):
        raw = pages.view(torch.uint8)[ids].view(pages.dtype) if pages.element_size() == 1 else pages[ids]
        x = raw.float().double()
        x = x if scale is None else x * scale.double().view(1, -1, 1, 1)
        got.append(x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :int(tree.node_len[n])])
    return got


def queries(tree, prefill):
    """(query row, path's K, path's V, visible keys) of every query."""
    row = 0
    for b, leaf in enumerate(tree.leaf_node):
        kv = [node_kv(tree, n) for n in tree.path(b)]
        k, v = (torch.cat([x[i] for x in kv], dim=1) for i in range(2))
        own = int(tree.node_len[leaf]) if prefill else 1
        for t in range(own):
            yield row, k, v, k.shape[1] - own + 1 + t if prefill else k.shape[1]
            row += 1


def capped(tree, cap, prefill=False):
    """(out, lse, bound of out, bound of lse), 64 bits.

    A row's logit s = cap tanh(x), x = scale <q, k> / cap, comes off by at most
      delta = 2^-16 A + 2^-20 min(cap, |s|max) + 2^-20,  A = max_t scale sum |q_i k_ti|:
    the fp32 sums of d <= 128 products (in chains of 16, whatever their order:
    under 130 roundings of 2^-24 A; twice that for the scale's factors), the
    tanh's own few units, and the exponent's sum and power of two (x up to
    cap / ln 2 rounds to 2^-24 of itself).  Weights are then off by 2 delta
    relative (their own and the sum's), P rounds to half a step, and the sums of
    n terms by n / 8 + 20 fp32 roundings (8 or more lanes or registers share a
    row's terms in every kernel)."""
    h_q, g = tree.num_q_heads, tree.group
    scale = tree.sm_scale or 1.0 / math.sqrt(tree.head_dim)
    out = torch.zeros(tree.q.shape, dtype=torch.float64, device=tree.q.device)
    lse = torch.full(tree.q.shape[:2], -math.inf, dtype=torch.float64, device=tree.q.device)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for row, k, v, n in queries(tree, prefill):
        if n == 0:
            continue
        q = tree.q[row].double().view(-1, g, tree.head_dim)
        kk, vv = k[:, :n], v[:, :n]
        s = torch.matmul(q, kk.transpose(1, 2)) * scale
        if cap:
            s = cap * torch.tanh(s / cap)
        big = (torch.matmul(q.abs(), kk.abs().transpose(1, 2)) * scale).amax(dim=-1)
        z = torch.logsumexp(s, dim=-1)
        p = torch.exp(s - z.unsqueeze(-1))
        delta = 2.0 ** -16 * big + 2.0 ** -20 * s.abs().amax(dim=-1) + 2.0 ** -20
        sums = (n / 8 + 20) * 2.0 ** -24
        o, mass = torch.matmul(p, vv), torch.matmul(p, vv.abs())
        out[row], lse[row] = o.reshape(h_q, -1), z.reshape(h_q)
        off = mass * (P_HALF[tree.mode] + 2 * sums + 2 * delta.unsqueeze(-1))
        tol_o[row] = (off + OUT_HALF[tree.mode] * (o.abs() + off) + 2.0 ** -126).reshape(h_q, -1)
        # (the result's own rounding: 2^-23 of it)
        tol_l[row] = (delta + sums + 2.0 ** -22 * z.abs()).reshape(h_q)
    return out, lse, tol_o, tol_l


def check(tree, cap, out, lse, prefill=False):
    ref_o, ref_l, tol_o, tol_l = capped(tree, cap, prefill)
    worst = ((out.double() - ref_o).abs() / tol_o.clamp(min=1e-300)).max()
    assert ((out.double() - ref_o).abs() <= tol_o).all(), f"out: {float(worst):.2f} of its bound"
    live = ref_l > -math.inf
    worst = ((lse.double() - ref_l)[live].abs() / tol_l[live]).max() if live.any() else 0
    assert ((lse.double() - ref_l)[live].abs() <= tol_l[live]).all(), f"lse: {float(worst):.2f} of its bound"
    assert (lse[~live] == -math.inf).all() and (out[~live] == 0).all()
