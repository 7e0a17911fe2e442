"""A layer served over a 4-bit cache: slots on the device, normed and rotated rows
written through them, prefill and decode over what was written; and long pieces."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import HeadNorm, Plan, kv_read, kv_scales, kv_slots, kv_write
from tests import fp4_ref as F
from tests import kv_ref as R
from tests import norm_ref as N

pytestmark = pytest.mark.gpu
H_Q, H_KV, D, PAGES = 8, 2, 128, 64


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def projected(gen, tokens):
    x = torch.randn((tokens, (H_Q + 2 * H_KV) * D), generator=gen, device="cuda").to(torch.bfloat16)
    return (y.unflatten(1, (-1, D)) for y in x.split([H_Q * D, H_KV * D, H_KV * D], dim=1))


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_layer_served():
    gen = R.generator(41)
    rotary, table = R.rotary_of((128, 1, False))
    w = [N.weight(gen, (D,), torch.bfloat16) for _ in range(2)]
    norm = HeadNorm(*w)
    pools = [F.random_pool(gen, PAGES, H_KV, 0, 255) for _ in range(2)]         # random bytes, NaN among them
    order = np.random.default_rng(4).permutation(PAGES).astype(np.int32)
    free, used = torch.from_numpy(order).cuda(), ints(0)
    prompt = 197
    # scales: of the normed keys, taken from a bf16 cache
    q, k, v = projected(gen, prompt)
    plain = [torch.empty((13, H_KV, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    slots = torch.arange(prompt, dtype=torch.int32, device="cuda")
    kv_write(k, v, *plain, slots, norm=HeadNorm(k_weight=w[1]))
    ks, vs = kv_scales(*kv_read(*plain, slots), rotary=rotary, mode="fp4")
    scales = dict(k_scale=1.2 * ks, v_scale=1.2 * vs)

    def write(q, k, v, slots, positions):
        out = kv_write(k, v, *pools, slots, q=q, norm=norm, rotary=rotary, positions=positions, **scales)
        ref, size = N.rows(q, w[0], rotary, table, positions)
        off = N.loose(ref, size)
        assert ((out.double() - ref).abs() <= off + R.HALF[torch.bfloat16] * (ref.abs() + off)).all()
        # what the cache holds: within a step of the block's scale
        ref, size = N.rows(k, w[1], rotary, table, positions)
        got = [F.decoded(p, s)[slots.long() // 16, :, slots.long() % 16] for p, s in zip(pools, scales.values())]
        for x, want in ((got[0], ref), (got[1], v.double())):
            most = want.unflatten(-1, (-1, 16)).abs().amax(dim=-1, keepdim=True)
            # half a step at the top (1 of 6) with the scale off by half a step of e4m3 (2^-4)
            assert ((x - want).unflatten(-1, (-1, 16)).abs() <= most / 6 * (1 + 2.0 ** -3)).all()
        return out

    def tree(parent, lens, pages, leaves, q):
        ptr = np.concatenate([[0], np.cumsum([len(p) for p in pages])]).astype(np.int32)
        return W.ForkTree(name="served", num_q_heads=H_Q, num_kv_heads=H_KV, head_dim=D, mode="fp4",
                          parent=np.array(parent, np.int32), node_len=np.array(lens, np.int32), node_page_ptr=ptr,
                          page_ids=np.concatenate(pages).astype(np.int32), leaf_node=np.array(leaves, np.int32),
                          num_physical_pages=PAGES, q=q, k_pages=pools[0], v_pages=pools[1], **scales)

    # the prompt: one sequence, pages from the list
    prompt_table = torch.full((1, 13), -1, dtype=torch.int32, device="cuda")
    slots, positions = kv_slots(prompt_table, ints(0), ints(prompt), prompt, free_pages=free, free_used=used, used_out=used)
    assert int(used) == 13 and prompt_table.tolist() == [order[:13].tolist()]
    q_out = write(q, k, v, slots, positions)
    t = tree([-1], [prompt], [order[:13]], [0], q_out)
    with Plan.for_prefill(t) as plan:
        out, lse = plan.decode_tree(t)
        plan.check()
    F.check(t, out, lse, prefill=True)

    # three threads open with a few tokens each, then go on step by step in place
    lens = [1, 16, 30]
    threads = torch.full((3, 8), -1, dtype=torch.int32, device="cuda")
    held, first = ints(0, 0, 0), ints(prompt, prompt, prompt)
    q, k, v = projected(gen, sum(lens))
    slots, positions = kv_slots(threads, held, ints(*lens), sum(lens), first=first, free_pages=free, free_used=used,
                                lens_out=held, used_out=used)
    assert held.tolist() == lens and int(used) == 17
    write(q, k, v, slots, positions)
    mine = [list(order[13:14]), list(order[14:15]), list(order[15:17])]
    t = tree([-1, 0, 0, 0], [prompt] + lens, [order[:13]] + mine, [1, 2, 3],
             torch.zeros((3, H_Q, D), dtype=torch.bfloat16, device="cuda"))
    taken = 17
    slots, positions = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2))
    step_slots = torch.cuda.CUDAGraph()
    with torch.cuda.graph(step_slots):
        kv_slots(threads, held, first=first, free_pages=free, free_used=used, slots=slots, positions=positions,
                 lens_out=held, used_out=used)
    with Plan.for_tree(t) as plan:
        for step in range(20):
            opened = []
            for i in range(3):                           # the host's own account of the list
                opened.append(-1)
                if lens[i] % 16 == 0:
                    opened[i] = int(order[taken])
                    mine[i].append(opened[i])
                    taken += 1
                lens[i] += 1
            plan.append(opened)
            q, k, v = projected(gen, 3)
            step_slots.replay()
            assert held.tolist() == lens and int(used) == taken
            q_out = write(q, k, v, slots, positions)
            t = tree([-1, 0, 0, 0], [prompt] + lens, [order[:13]] + mine, [1, 2, 3], q_out)
            out, lse = plan.decode_tree(t)
            plan.check()
            F.check(t, out, lse)


def test_long_pieces():
    """Pieces of many stages (several windows of page rows): 64 requests of 6000 to 8000 tokens,
    the first and the last of them against 64 bits."""
    lens = [int(x) for x in np.random.default_rng(7).integers(6000, 8001, 64)]
    shape = W.build_tree("long", [-1] * 64, lens, list(range(64)), num_q_heads=8, num_kv_heads=8, head_dim=D,
                         mode="fp4", seed=3, permute_pages=True, values=False)
    gen = R.generator(5)
    q = torch.randn((64, 8, D), generator=gen, device="cuda").to(torch.bfloat16)
    pools = [F.random_pool(gen, shape.num_physical_pages, 8) for _ in range(2)]
    scales = [0.3 + 0.5 * torch.rand(8, generator=gen, device="cuda") for _ in range(2)]
    t = replace(shape, q=q, k_pages=pools[0], v_pages=pools[1], k_scale=scales[0], v_scale=scales[1])
    with Plan.for_tree(t) as plan:
        assert max(plan.export(0)[:, 1]) > 60            # pages of an item
        out, lse = plan.decode_tree(t)
        plan.check()
    for b in (0, 31, 63):
        ids = t.page_ids[t.node_page_ptr[b]:t.node_page_ptr[b + 1]]
        one = replace(t, parent=np.array([-1], np.int32), node_len=t.node_len[b:b + 1],
                      node_page_ptr=np.array([0, len(ids)], np.int32), page_ids=np.arange(len(ids), dtype=np.int32),
                      leaf_node=np.array([0], np.int32), num_physical_pages=len(ids), q=q[b:b + 1],
                      k_pages=pools[0][ids.tolist()], v_pages=pools[1][ids.tolist()])
        F.check(one, out[b:b + 1], lse[b:b + 1])


def test_pages_past_4_gb():
    """Pages whose bytes lie more than 2^32 into a pool: written, read, decoded and prefilled as
    in a small pool."""
    pages, heads = 480_000, 8                            # 4.4 GB each
    gen = R.generator(11)
    small = [torch.zeros((40, heads, 9 * D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    large = [torch.empty((pages, heads, 9 * D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    last = torch.arange(pages - 40, pages, device="cuda")
    for x in large:
        x[last] = 0
    tokens = 600
    k, v = (torch.randn((tokens, heads, D), generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    scales = dict(k_scale=torch.full((heads,), 1e-3, device="cuda"), v_scale=torch.full((heads,), 1e-3, device="cuda"))
    slots = torch.randperm(640, generator=gen, device="cuda")[:tokens].int()
    far = slots + 16 * (pages - 40)
    kv_write(k, v, *small, slots, **scales)
    kv_write(k, v, *large, far, **scales)
    assert all(torch.equal(x[last], y) for x, y in zip(large, small))
    assert all(torch.equal(x, y) for x, y in zip(kv_read(*large, far, **scales), kv_read(*small, slots, **scales)))
    kw = dict(num_q_heads=32, num_kv_heads=heads, head_dim=D, mode="fp4", parent=[-1, 0, 0, 0, 0, 0], sm_scale=0.1,
              node_len=[330, 40, 64, 17, 50, 9], node_page_ptr=[0, 21, 24, 28, 30, 34, 35])
    for prefill in (False, True):
        out = []
        for pools, first in ((small, 0), (large, pages - 40)):
            ids = (torch.arange(35) * 11 % 40 + first).tolist()
            with Plan(page_ids=ids, leaf_node=[1, 2, 3, 4, 5], num_physical_pages=pools[0].shape[0], prefill=prefill,
                      **kw) as plan:
                q = torch.randn((plan.num_leaves, 32, D), generator=R.generator(2), device="cuda").to(torch.bfloat16)
                out.append(plan.decode(q, *pools, **scales))
                plan.check()
        assert out[0][0].isfinite().all() and out[0][0].abs().max() > 0.01
        assert all(torch.equal(x, y) for x, y in zip(*out))
