"""A NaN score makes its row's out and lse NaN, in every merge and epilogue: also
where every score of the row is NaN, which no running maximum shows."""
import math

import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan, lse_merge
from tests import cap_ref as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def run(tree, cap, prefill=False):
    make = Plan.for_prefill if prefill else Plan.for_tree
    with make(tree, logit_cap=cap) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
        return out, lse, plan.launches_per_decode()


def check(tree, cap, out, lse, rows, prefill=False):
    """NaN in all of `rows` rows of heads, the others as near as ever."""
    ref_o, ref_l, tol_o, tol_l = C.capped(tree, cap, prefill)
    lost = ref_l.isnan()
    assert int(lost.sum()) == rows
    assert out[lost].isnan().all(), f"{int((~out[lost].isnan()).sum())} finite elements"
    assert lse[lost].isnan().all(), lse[lost][~lse[lost].isnan()][:4].tolist()
    assert ((out.double() - ref_o).abs() <= tol_o)[~lost].all()
    live = ~lost & (ref_l > -math.inf)
    assert ((lse.double() - ref_l).abs() <= tol_l)[live].all()
    assert (lse[ref_l == -math.inf] == -math.inf).all()


def spoil(tree, node, tokens, head):
    """One element of these keys of a node becomes NaN."""
    for t in tokens:
        page = int(tree.page_ids[int(tree.node_page_ptr[node]) + t // 16])
        if tree.mode == "fp8":
            tree.k_pages.view(torch.uint8)[page, head, t % 16, 5] = 0x7F
        else:
            tree.k_pages[page, head, t % 16, 5] = math.nan


CAPS = [0.0, 50.0, 90.0]

# (branches, heads, prefix, own): rows of 4, 2 and 1 warps, and of a group's one warp, in the merge
MERGES = {"four": (6, (8, 2), 300, 40), "two": (100, (16, 2), 130, 20), "one": (150, (32, 4), 130, 20),
          "pair": (1100, (8, 4), 60, 20), "quad": (1100, (16, 4), 60, 20), "short": (6, (8, 2), 0, 9)}


def forest(mode, case, d=128):
    leaves, (h_q, h_kv), prefix, own = MERGES[case]
    return W.build_tree("nan", [-1] + [0] * leaves, [prefix] + [own + i % 7 for i in range(leaves)],
                        list(range(1, leaves + 1)), num_q_heads=h_q, num_kv_heads=h_kv, head_dim=d, mode=mode,
                        seed=3, device="cuda", tail_value=math.nan)


@pytest.mark.parametrize("case,mode,d,cap", [
    (case, mode, d, cap) for case in ("four", "short")
    for mode, d in (("bf16", 128), ("fp8", 128), ("fp32", 128)) for cap in CAPS] + [
    (case, mode, d, cap) for case in ("two", "one") for mode, d, cap in (("bf16", 64, 50.0), ("fp32", 64, 0.0))] + [
    ("pair", "bf16", 128, 90.0), ("quad", "fp32", 128, 0.0)])
def test_decode(case, mode, d, cap):
    """One branch's last key; every key of a branch's path; a query."""
    leaves, (h_q, h_kv), prefix, own = MERGES[case]
    group = h_q // h_kv
    one, whole, query = (forest(mode, case, d) for _ in range(3))
    spoil(one, 3, [own + 2 % 7 - 1], 1)
    check(one, cap, *run(one, cap)[:2], group)
    spoil(whole, 0, range(prefix), 1)
    spoil(whole, 5, range(own + 4 % 7), 1)
    check(whole, cap, *run(whole, cap)[:2], group * (leaves if prefix else 1))
    if mode != "fp8":                                # (narrowed to f16 there, under rules of its own)
        query.q[2, 1] = math.nan
        check(query, cap, *run(query, cap)[:2], 1)


PREFILLS = {"direct": ([-1, 0, 0], [60, 64, 70], [1, 2]), "merged": ([-1, 0, 0], [9000, 130, 30], [1, 2]),
            "root": ([-1], [90], [0])}


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
@pytest.mark.parametrize("case", sorted(PREFILLS))
@pytest.mark.parametrize("cap", CAPS)
def test_prefill(mode, case, cap):
    parent, lens, chunks = PREFILLS[case]

    def tree():
        return W.build_prefill("nanp", parent, lens, chunks, num_q_heads=8, num_kv_heads=2, head_dim=128, mode=mode,
                               seed=4, device="cuda", tail_value=math.nan)
    one, whole = tree(), tree()
    spoil(one, chunks[-1], [17], 1)
    out, lse, launches = run(one, cap, True)
    assert launches == (2 if case == "merged" else 1)           # (both ways to the result are met)
    check(one, cap, out, lse, (lens[chunks[-1]] - 17) * 4, True)
    for n in range(len(lens)):
        spoil(whole, n, range(lens[n]), 0)
    check(whole, cap, *run(whole, cap, True)[:2], whole.q.shape[0] * 4, True)
    if mode == "bf16":
        query = tree()
        query.q[5, 2] = math.nan
        check(query, cap, *run(query, cap, True)[:2], 1, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lse_merge(dtype):
    """A NaN row stays NaN beside a finite one, an empty one and another of its kind."""
    o = torch.ones((7, 128), dtype=dtype, device="cuda")
    a = torch.tensor([math.nan, 1.0, math.nan, -math.inf, math.nan, -math.inf, 0.5], device="cuda")
    b = torch.tensor([1.0, math.nan, -math.inf, math.nan, math.nan, -math.inf, 0.5], device="cuda")
    oa, ob = o.clone(), o.clone()
    oa[a.isnan()], ob[b.isnan()] = math.nan, math.nan
    oa[a == -math.inf], ob[b == -math.inf] = 0.0, 0.0
    out, lse = lse_merge(oa, a, ob, b)
    assert out[:5].isnan().all() and lse[:5].isnan().all()
    assert (out[5] == 0).all() and lse[5] == -math.inf
    assert (out[6] == 1).all() and abs(float(lse[6]) - 0.5 - math.log(2.0)) <= 2.0 ** -22


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_halves_of_a_nan_row_meet(mode):
    """What lse_merge gets from two plans over disjoint keys, of a NaN query."""
    whole = W.build_tree("w", [-1, 0], [96, 50], [1], num_q_heads=8, num_kv_heads=2, head_dim=128, seed=2,
                         device="cuda", mode=mode)
    whole.q[0, 3] = math.nan
    parts = []
    for n in (0, 1):
        ids = whole.page_ids[whole.node_page_ptr[n]:whole.node_page_ptr[n + 1]]
        with Plan(num_q_heads=8, num_kv_heads=2, head_dim=128, mode=mode, parent=[-1], node_len=whole.node_len[n:n + 1],
                  node_page_ptr=[0, len(ids)], page_ids=ids, leaf_node=[0],
                  num_physical_pages=whole.num_physical_pages) as plan:
            parts.append(plan.decode(whole.q, whole.k_pages, whole.v_pages))
            plan.check()
    out, lse = lse_merge(*parts[0], *parts[1])
    lost = torch.arange(8, device="cuda") == 3
    assert out[0, lost].isnan().all() and lse[0, lost].isnan().all()
    assert out[0, ~lost].isfinite().all() and lse[0, ~lost].isfinite().all()
