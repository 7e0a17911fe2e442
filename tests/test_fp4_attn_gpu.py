"""Decode and prefill over a 4-bit cache against 64-bit attention over what the
bytes stand for: head layouts, trees, page edges, caps, updates, NaN."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300.api import ParasonError, Plan
from tests import fp4_ref as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def decode(t, cap=0.0, prefill=False):
    with Plan.for_tree(t, prefill=prefill, logit_cap=cap) as plan:
        out, lse = plan.decode_tree(t)
        plan.check()
    F.check(t, out, lse, prefill, cap)
    return out, lse


FLAT = ([-1, 0, 0, 0, 0], [100, 17, 64, 1, 33], [1, 2, 3, 4])
NESTED = ([-1, 0, 0, 1, 1, 2, 2, 2], [70, 33, 5, 16, 40, 1, 15, 31], [3, 4, 5, 6, 7])
REQUESTS = ([-1, 0, 0, -1, 3, 3], [48, 20, 7, 129, 64, 2], [1, 2, 4, 5])
EMPTY = ([-1, 0, 1, 0, -1], [0, 20, 35, 0, 0], [2, 3, 4])


@pytest.mark.parametrize("tree", [FLAT, NESTED, REQUESTS, EMPTY])
@pytest.mark.parametrize("heads", [(8, 2), (5, 1), (16, 16), (12, 2), (7, 1), (32, 2)])
def test_decode(tree, heads):
    decode(F.tree_of(*tree, *heads, seed=sum(heads)))


@pytest.mark.parametrize("tokens", [1, 2, 3, 15, 16, 17, 31, 32, 33, 100, 1000, 5000])
@pytest.mark.parametrize("heads", [(8, 1), (2, 1)])
def test_one_branch(tokens, heads):
    decode(F.tree_of([-1], [tokens], [0], *heads, seed=tokens))


@pytest.mark.parametrize("prefix", [1, 16, 63, 64, 65, 200, 1500])
def test_shared_prefix_tiles(prefix):
    """More than 16 rows under one node: the tensor-core tile, one and several row tiles."""
    decode(F.tree_of([-1] + [0] * 12, [prefix] + list(range(5, 17)), list(range(1, 13)), 16, 2, seed=prefix))
    decode(F.tree_of([-1] + [0] * 45, [prefix] + [3] * 45, list(range(1, 46)), 8, 2, seed=prefix + 1))


def test_long_prefix_and_branches():
    lens = [9000] + [int(x) for x in np.random.default_rng(0).integers(1, 2500, 20)]
    decode(F.tree_of([-1] + [0] * 20, lens, list(range(1, 21)), 32, 4, seed=3))


def test_sharp_scores_and_scale():
    decode(F.tree_of(*NESTED, 8, 2, seed=5, q_std=6.0))
    decode(F.tree_of(*NESTED, 8, 2, seed=6, q_std=3.0, sm_scale=0.3))


@pytest.mark.parametrize("cap", [2.0, 50.0, 300.0])
def test_capped(cap):
    decode(F.tree_of(*NESTED, 16, 2, seed=7, q_std=4.0), cap)
    decode(F.tree_of([-1] + [0] * 20, [300] + [9] * 20, list(range(1, 21)), 8, 2, seed=8, q_std=4.0), cap)
    decode(F.tree_of([-1, 0, 0], [77, 40, 130], [1, 2], 8, 2, seed=9, prefill=True, q_std=4.0), cap, prefill=True)


PREFILL = {
    "join": ([-1, 0, 0, 0, 1], [300, 70, 33, 64, 41], [2, 3, 4], 8, 2),
    "root": ([-1], [200], [0], 8, 2),
    "edges": ([-1, 0, 0, 0, 0, 0, 0], [17, 1, 15, 16, 63, 64, 65], [1, 2, 3, 4, 5, 6], 8, 2),
    "g1": ([-1, 0, 1], [50, 90, 130], [2], 4, 4),
    "g16": ([-1, 0, 0], [77, 40, 9], [1, 2], 32, 2),
    "g7": ([-1, 0, 1, 1], [33, 21, 70, 5], [2, 3], 7, 1),
    "chain": ([-1, 0, 1, 2, 3], [129, 1, 47, 90, 77], [4], 8, 2),
    "long": ([-1, 0], [1300, 300], [1], 16, 4),
    "empty": ([-1, 0, 1, 0], [0, 20, 35, 0], [2, 3], 8, 2),
    "one_token": ([-1, 0], [5, 1], [1], 8, 2),
}


@pytest.mark.parametrize("name", sorted(PREFILL))
def test_prefill(name):
    parent, lens, leaves, h_q, h_kv = PREFILL[name]
    decode(F.tree_of(parent, lens, leaves, h_q, h_kv, seed=len(name), prefill=True), prefill=True)


@pytest.mark.parametrize("extreme", ["zero", "most", "subnormal"])
def test_block_scales_at_the_ends(extreme):
    """Scales of 0, the largest (448) and e4m3's subnormals, in every second block."""
    t = F.tree_of(*FLAT, 8, 2, seed=11)
    for p, s in ((t.k_pages, t.k_scale), (t.v_pages, t.v_scale)):
        scales = F.split(p)[1]
        held = scales != F.NAN_SCALE
        code = {"zero": 0, "most": 0x7E, "subnormal": 3}[extreme]
        pick = torch.zeros_like(held)
        pick[..., ::2] = True
        scales[held & pick] = code
        if extreme == "most":
            s *= 2.0 ** -9
    decode(t)


def test_append_and_fork():
    parent, lens, leaves = [-1, 0, 0], [90, 30, 17], [1, 2]
    t = F.tree_of(parent, lens, leaves, 8, 2, seed=12, extra_pages=8, permute=False)
    used = int(t.node_page_ptr[-1])
    gen = torch.Generator(device="cuda").manual_seed(1)
    fresh = [F.random_pool(gen, t.num_physical_pages, 2) for _ in range(2)]
    pools = [p.clone() for p in (t.k_pages, t.v_pages)]
    for a, b in zip(pools, fresh):                       # tokens to come have values too
        a.copy_(torch.where(F_held(t), a, b))
    ids = [list(t.page_ids[t.node_page_ptr[n]:t.node_page_ptr[n + 1]]) for n in range(3)]
    with Plan.for_tree(t) as plan:
        for step in range(20):
            opened = [-1, -1]
            for i, n in enumerate(leaves):
                if lens[n] % 16 == 0:
                    opened[i] = used
                    ids[n].append(used)
                    used += 1
                lens[n] += 1
            plan.append(opened)
        child = [5, 20]
        pages = [[used], [used + 1, used + 2]]
        plan.fork(0, child, pages)
        parent, lens, ids = parent + [1, 1], lens + child, ids + pages
        ptr = np.concatenate([[0], np.cumsum([len(p) for p in ids])]).astype(np.int32)
        q = torch.randn((3, 8, 128), generator=gen, device="cuda").to(torch.bfloat16)
        grown = replace(t, parent=np.array(parent, np.int32), node_len=np.array(lens, np.int32), node_page_ptr=ptr,
                        page_ids=np.array(sum(ids, []), np.int32), leaf_node=np.array([3, 2, 4], np.int32), q=q,
                        k_pages=pools[0], v_pages=pools[1])
        out, lse = plan.decode(q, *pools, k_scale=t.k_scale, v_scale=t.v_scale)
        plan.check()
    F.check(grown, out, lse)


def F_held(t):
    """Bytes of the pool that hold tokens."""
    scales = F.split(t.k_pages)[1] != F.NAN_SCALE
    values = scales.repeat_interleave(F.D // 2 // (F.D // 16), dim=-1)
    return torch.cat([values.flatten(2), scales.flatten(2)], dim=2)


def test_shards():
    t = F.tree_of(*REQUESTS, 8, 2, seed=13)
    want = decode(t)
    for rank in range(2):
        with Plan.for_tree(t, shard=(_lib.SHARD_REQUESTS, rank, 2)) as plan:
            rows = plan.export(_lib.TABLE_SHARD_BRANCHES)
            out, lse = plan.decode(t.q[rows.tolist()].contiguous(), t.k_pages, t.v_pages, k_scale=t.k_scale,
                                   v_scale=t.v_scale)
            plan.check()
        F.check(replace(t, leaf_node=t.leaf_node[rows], q=t.q[rows.tolist()].contiguous()), out, lse)
        with Plan.for_tree(t, shard=(_lib.SHARD_KV_HEADS, rank, 2)) as plan:
            part = [p[:, rank:rank + 1].contiguous() for p in (t.k_pages, t.v_pages)]
            scales = [s[rank:rank + 1].contiguous() for s in (t.k_scale, t.v_scale)]
            q = t.q[:, 4 * rank:4 * rank + 4].contiguous()
            out, lse = plan.decode(q, *part, k_scale=scales[0], v_scale=scales[1])
            plan.check()
        F.check(replace(t, num_q_heads=4, num_kv_heads=1, q=q, k_pages=part[0], v_pages=part[1], k_scale=scales[0],
                        v_scale=scales[1]), out, lse)
    assert torch.isfinite(want[1]).all()


def test_without_a_workspace_and_again():
    t = F.tree_of(*NESTED, 8, 2, seed=14)
    with Plan.for_tree(t) as plan:
        out, lse = plan.decode_tree(t)
        again, _ = plan.decode_tree(t)
        third = torch.empty_like(out)
        plan.decode_no_alloc(t.q, t.k_pages, t.v_pages, third, None, k_scale=t.k_scale, v_scale=t.v_scale)
        plan.check()
    assert torch.equal(out, again) and torch.equal(out, third)


def test_captured_on_a_stream():
    """A captured decode replays over what the pools, q and scales hold then."""
    t = F.tree_of(*NESTED, 8, 2, seed=15)
    other = F.tree_of(*NESTED, 8, 2, seed=15)
    gen = torch.Generator(device="cuda").manual_seed(9)
    with Plan.for_tree(t) as plan:
        out, lse = plan.decode_tree(t)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            plan.decode_tree(t, out=out, lse=lse)
        t.q.copy_(torch.randn(t.q.shape, generator=gen, device="cuda"))
        t.k_scale.mul_(0.5)
        F.split(t.v_pages)[0].copy_(torch.where(F.split(t.v_pages)[1].repeat_interleave(8, -1) == F.NAN_SCALE,
                                                F.split(t.v_pages)[0], F.split(other.v_pages)[0].flip(0)))
        graph.replay()
        plan.check()
    F.check(t, out, lse)


def test_nan_scale_reaches_who_sees_it():
    t = F.tree_of([-1, 0, 0], [40, 20, 20], [1, 2], 8, 2, seed=16)
    page = int(t.page_ids[t.node_page_ptr[1]])
    F.split(t.v_pages)[1][page, 0, 3, 2] = F.NAN_SCALE            # branch 0, kv head 0, elements 32..47
    with Plan.for_tree(t) as plan:
        out, lse = plan.decode_tree(t)
        plan.check()
    bad = torch.isnan(out)
    assert bad[0, :4, 32:48].all() and bad.sum() == 4 * 16 and torch.isfinite(lse).all()


def test_q_beyond_f16_is_reported():
    t = F.tree_of(*FLAT, 8, 2, seed=17)
    t.q[2, 3, 5] = 70000.0
    with Plan.for_tree(t) as plan:
        plan.decode_tree(t)
        with pytest.raises(ParasonError) as e:
            plan.check()
    assert e.value.status == _lib.ERANGE


def test_wrong_pools():
    t = F.tree_of(*FLAT, 8, 2, seed=18)
    with Plan.for_tree(t) as plan:
        for k in (t.k_pages[:, :, :-9].contiguous(), t.k_pages.view(torch.int8), t.k_pages[:-1],
                  t.k_pages.unflatten(2, (16, 72))):
            with pytest.raises(ValueError):
                plan.decode(t.q, k, t.v_pages, k_scale=t.k_scale, v_scale=t.v_scale)
        with pytest.raises(ValueError):
            plan.decode(t.q, t.k_pages, t.v_pages, k_scale=t.k_scale)


def test_pinned_q_and_results():
    """q read from, and out and lse written to, pinned host memory; then through the binding's own checks."""
    t = F.tree_of(*NESTED, 24, 2, seed=17)
    with Plan.for_tree(t) as plan:
        out, lse = plan.decode_tree(t)
        there, lse_there = plan.decode(t.q.cpu().pin_memory(), t.k_pages, t.v_pages, k_scale=t.k_scale, v_scale=t.v_scale)
        torch.cuda.synchronize()
        plan.check()
        assert there.is_pinned() and torch.equal(there, out.cpu()) and torch.equal(lse_there, lse.cpu())
        for bad in (t.q.float(), t.q[:-1], t.q.cpu(), t.q.transpose(1, 2).contiguous().transpose(1, 2)):
            with pytest.raises(ValueError):
                plan.decode(bad, t.k_pages, t.v_pages, k_scale=t.k_scale, v_scale=t.v_scale)
        for bad in (t.k_scale[:1], t.k_scale.double(), t.k_scale.cpu()):
            with pytest.raises(ValueError):
                plan.decode(t.q, t.k_pages, t.v_pages, k_scale=bad, v_scale=t.v_scale)
