"""Capped logits in every attention kernel against 64-bit arithmetic: caps far
above, at and far below the scores, tiles of every kind, after updates, and in
a replayed graph."""
import math

import pytest
import torch

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan, lse_merge
from tests import cap_ref as C
from tests import parity as PT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def decode(tree, cap, **kw):
    with Plan.for_tree(tree, logit_cap=cap, **kw) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    return out, lse


def forest(seed, mode, h_q, h_kv, d, q_std=1.0, **kw):
    kw = dict(dict(tail_value=math.nan), **kw)
    return PT.nan_fill_unused_pages(W.random_tree(seed, mode=mode, h_q=h_q, h_kv=h_kv, d=d, q_std=q_std,
                                                  device="cuda", **kw))


# (mode, q heads, kv heads, head_dim): 16-row and transposed suffix steps, both
# head dims, e4m3, fp32; wide nodes run on the tcgen05 tile
SHAPES = [("bf16", 8, 2, 64), ("bf16", 8, 2, 128), ("bf16", 16, 2, 128), ("bf16", 4, 4, 128), ("bf16", 32, 2, 128),
          ("bf16", 12, 2, 64), ("fp8", 8, 2, 128), ("fp8", 16, 2, 128), ("fp8", 3, 3, 128), ("fp32", 8, 2, 128),
          ("fp32", 16, 1, 64), ("fp32", 5, 5, 128)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("cap,q_std", [(50.0, 1.0), (30.0, 8.0), (2.0, 4.0), (2.0 ** -10, 1.0), (2.0 ** 20, 1.0),
                                       (1000.0, 30.0)])
def test_decode(shape, cap, q_std):
    mode, h_q, h_kv, d = shape
    tree = forest(21, mode, h_q, h_kv, d, q_std)
    C.check(tree, cap, *decode(tree, cap))


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("cap,q_std", [(50.0, 1.0), (20.0, 10.0)])
def test_wide_tiles(mode, cap, q_std):
    """Pairs of row tiles (bf16), single tiles (e4m3), fp32's 16-row tiles."""
    tree = W.pair_fixture(mode=mode, device="cuda", q_std=q_std)
    C.check(tree, cap, *decode(tree, cap))


@pytest.mark.parametrize("d", [64, 128])
def test_single_tcgen05_tile(d):
    tree = W.build_tree("tile", [-1] + [0] * 9, [777] + [5] * 9, list(range(1, 10)), num_q_heads=8, num_kv_heads=2,
                        head_dim=d, seed=5, q_std=6.0, device="cuda", tail_value=math.nan)
    C.check(tree, 25.0, *decode(tree, 25.0))


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
@pytest.mark.parametrize("seed", range(6))
def test_random_forests(mode, seed):
    h_q, h_kv = [(8, 2), (28, 4), (16, 16), (64, 8), (6, 1), (32, 2)][seed]
    tree = forest(seed, mode, h_q, h_kv, 128, 3.0, depth=1 + seed % 3, len_range=(0, 200), leaf_min_len=0)
    C.check(tree, 15.0, *decode(tree, 15.0))


def test_empty_paths():
    tree = W.build_tree("empty", [-1, 0, 0], [0, 0, 7], [1, 2], num_q_heads=4, num_kv_heads=2, head_dim=128,
                        device="cuda")
    out, lse = decode(tree, 30.0)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    C.check(tree, 30.0, out, lse)


PREFILLS = {
    "join": ([-1, 0, 0, 0, 1], [300, 70, 33, 64, 41], [2, 3, 4], 8, 2),
    "root": ([-1], [200], [0], 8, 2),
    "edges": ([-1, 0, 0, 0, 0, 0, 0], [17, 1, 15, 16, 63, 64, 65], [1, 2, 3, 4, 5, 6], 8, 2),
    "g1": ([-1, 0, 1], [50, 90, 130], [2], 4, 4),
    "g16": ([-1, 0, 0], [77, 40, 9], [1, 2], 32, 2),
    "one": ([-1, 0], [40, 1], [1], 4, 4),
    "empty": ([-1, 0, 1, 0], [0, 20, 35, 0], [2, 3], 8, 2),
    # a long path in several pieces (partials and a merge)
    "pieces": ([-1, 0, 0], [9000, 130, 3], [1, 2], 4, 1),
}


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
@pytest.mark.parametrize("case", sorted(PREFILLS))
@pytest.mark.parametrize("cap,q_std", [(50.0, 1.0), (10.0, 8.0)])
def test_prefill(mode, case, cap, q_std):
    parent, lens, chunks, h_q, h_kv = PREFILLS[case]
    tree = W.build_prefill(case, parent, lens, chunks, num_q_heads=h_q, num_kv_heads=h_kv, head_dim=128, mode=mode,
                           seed=3, q_std=q_std, device="cuda", permute_pages=True, extra_pages=6, tail_value=math.nan)
    PT.nan_fill_unused_pages(tree)
    with Plan.for_prefill(tree, logit_cap=cap) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    C.check(tree, cap, out, lse, prefill=True)


def test_cap_on_and_off():
    """Without a cap the bits are those of a plan that never had one; a cap can be moved between calls."""
    for mode, h_q in (("bf16", 8), ("fp8", 16), ("fp32", 8)):
        tree = forest(4, mode, h_q, 2, 128, 4.0)
        plain = decode(tree, 0.0)
        with Plan.for_tree(tree) as plan:
            for cap in (0.0, 12.0, 40.0, 0.0):
                plan.set_logit_cap(cap)
                out, lse = plan.decode_tree(tree)
                plan.check()
                C.check(tree, cap, out, lse)
            assert torch.equal(out, plain[0]) and torch.equal(lse, plain[1])


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
def test_after_appends_and_a_fork(mode):
    tree = W.build_tree("grow", [-1, 0, 0, 0], [200, 31, 16, 2], [1, 2, 3], num_q_heads=8, num_kv_heads=2,
                        head_dim=128, mode=mode, seed=4, extra_pages=40, q_std=5.0, device="cuda")
    pool = W.free_pages(tree)
    with Plan.for_tree(tree, logit_cap=20.0) as plan:
        for _ in range(5):
            tree, new_pages = W.grow_branches(tree, pool)
            plan.append(new_pages)
        C.check(tree, 20.0, *plan.decode_tree(tree))
        tree, pages = W.fork_branch(tree, 1, [1, 20], pool)
        plan.fork(1, [1, 20], pages)
        C.check(tree, 20.0, *plan.decode_tree(tree))
        plan.check()


def test_no_alloc_and_shards():
    tree = forest(8, "bf16", 8, 2, 128, 5.0)
    want = decode(tree, 20.0)
    with Plan.for_tree(tree, logit_cap=20.0) as plan:
        out, lse = torch.empty_like(tree.q), torch.empty(tree.q.shape[:2], device="cuda")
        plan.decode_no_alloc(tree.q, tree.k_pages, tree.v_pages, out, lse)
        plan.check()
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    with Plan.for_tree(tree, logit_cap=20.0, shard=(_lib.SHARD_KV_HEADS, 1, 2)) as plan:
        out, lse = plan.decode(tree.q[:, 4:].contiguous(), tree.k_pages[:, 1:].contiguous(),
                               tree.v_pages[:, 1:].contiguous())
        plan.check()
    ref_o, ref_l, tol_o, tol_l = C.capped(tree, 20.0)
    assert ((out.double() - ref_o[:, 4:]).abs() <= tol_o[:, 4:]).all()
    assert ((lse.double() - ref_l[:, 4:]).abs() <= tol_l[:, 4:]).all()


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
def test_first_capped_call_is_captured(mode):
    """The cap's kernels are ready once the cap is set: the first capped call may be a captured one."""
    tree = forest(9, mode, 16, 2, 128, 6.0)
    with Plan.for_tree(tree) as plan:
        out, lse = plan.decode_tree(tree)                  # (uncapped)
        ws = plan.workspace(tree.q.device)
        torch.cuda.synchronize()
        plan.set_logit_cap(11.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan.decode_tree(tree, out=out, lse=lse, workspace=ws)
        plan.set_logit_cap(0.0)                            # the captured call keeps its own
        for _ in range(3):
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        plan.check()
        C.check(tree, 11.0, out, lse)


def test_merge_of_capped_halves():
    """lse_merge joins capped results over disjoint keys."""
    whole = W.build_tree("w", [-1, 0], [96, 50], [1], num_q_heads=8, num_kv_heads=2, head_dim=128, seed=2, q_std=8.0,
                         device="cuda", mode="fp32")
    parts = []
    for lo, hi in ((0, 1), (1, 2)):
        ids = whole.page_ids[whole.node_page_ptr[lo]:whole.node_page_ptr[hi]]
        with Plan(num_q_heads=8, num_kv_heads=2, head_dim=128, mode="fp32", parent=[-1],
                  node_len=whole.node_len[lo:hi], node_page_ptr=[0, len(ids)], page_ids=ids, leaf_node=[0],
                  num_physical_pages=whole.num_physical_pages, logit_cap=9.0) as plan:
            parts.append(plan.decode(whole.q, whole.k_pages, whole.v_pages))
            plan.check()
    out, lse = lse_merge(*parts[0], *parts[1])
    ref_o, ref_l, tol_o, tol_l = C.capped(whole, 9.0)
    # (each half carries its own bound, and the merge two fp32 roundings more)
    assert ((out.double() - ref_o).abs() <= 3 * tol_o).all()
    assert ((lse.double() - ref_l).abs() <= 3 * tol_l).all()


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
def test_small_scores_beside_large_ones(mode):
    """Rows whose scores stay far below the cap keep their own accuracy in a tile
    whose other rows are at the cap."""
    tree = W.build_tree("rows", [-1] + [0] * 8, [500] + [3] * 8, list(range(1, 9)), num_q_heads=8, num_kv_heads=2,
                        head_dim=128, mode=mode, seed=6, q_std=0.5, device="cuda")
    tree.q[1::2] *= 3000.0
    C.check(tree, 1000.0, *decode(tree, 1000.0))


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("cap", [50.0, 50.59, 50.61, 90.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_every_key_at_the_cap(mode, cap, sign):
    """All weights near e^cap, or near e^-cap: the mean of V, lse = ln n + s.  (50.6 is where the kernels go from
    sums of e^s to a running maximum.)"""
    tree = W.build_tree("sat", [-1, 0, 0, 0], [700, 33, 1, 100], [1, 2, 3], num_q_heads=16, num_kv_heads=2,
                        head_dim=128, mode=mode, seed=7, device="cuda", tail_value=math.nan)
    tree.q.fill_(8.0)
    if mode == "fp8":
        tree.k_pages.view(torch.uint8).copy_(torch.full_like(tree.k_pages.float(), 256.0 * sign).to(
            torch.float8_e4m3fn).view(torch.uint8))
    else:
        tree.k_pages.fill_(16.0 * sign)
    out, lse = decode(tree, cap)
    C.check(tree, cap, out, lse)
    # every key's logit: <q, k> = 128 * 8 * k (in e4m3 tanh is not quite 1 there)
    n = torch.tensor([733, 701, 800], device="cuda").double()[:, None]
    key = 256.0 * sign * tree.k_scale.double() if mode == "fp8" else torch.full((2,), 16.0 * sign, device="cuda").double()
    at = (cap * torch.tanh(128 * 8 * key / math.sqrt(128) / cap)).repeat_interleave(8)
    assert ((lse.double() - (n.log() + at)).abs() <= 2.0 ** -18 * (cap + n.log())).all()


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
def test_scores_past_fp32(mode):
    """A score that overflows to infinity is at the cap."""
    tree = W.build_tree("inf", [-1, 0, 0], [600, 40, 40], [1, 2], num_q_heads=16, num_kv_heads=2, head_dim=128,
                        mode=mode, seed=8, device="cuda")
    tree.q.fill_(2.0 ** 62)
    signs = torch.where(torch.arange(tree.k_pages.shape[2], device="cuda") % 3 == 0, -1.0, 1.0)
    tree.k_pages.copy_((2.0 ** 62 * signs).view(1, 1, -1, 1).expand_as(tree.k_pages))
    for cap in (20.0, 100.0):
        out, lse = decode(tree, cap)
        ref_o, ref_l, tol_o, tol_l = C.capped(tree, cap)
        # (the bound's A is infinite here: the logits are +-cap exactly)
        assert ((lse.double() - ref_l).abs() <= 2.0 ** -18 * ref_l.abs()).all()
        rel = ((out.double() - ref_o).norm() / ref_o.norm()).item()
        assert rel <= (2.0 ** -7 if mode == "bf16" else 2.0 ** -18)


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
def test_prefill_every_key_at_minus_the_cap(mode):
    tree = W.build_prefill("satp", [-1, 0], [300, 90], [1], num_q_heads=8, num_kv_heads=2, head_dim=128, mode=mode,
                           seed=9, device="cuda", tail_value=math.nan)
    tree.q.fill_(-8.0)
    if mode == "fp8":
        tree.k_pages.view(torch.uint8).copy_(torch.full_like(tree.k_pages.float(), 256.0).to(
            torch.float8_e4m3fn).view(torch.uint8))
    else:
        tree.k_pages.fill_(16.0)
    for cap in (50.0, 80.0):
        with Plan.for_prefill(tree, logit_cap=cap) as plan:
            out, lse = plan.decode_tree(tree)
            plan.check()
        C.check(tree, cap, out, lse, prefill=True)


def nan_key(tree, node, token, head):
    """One element of a key becomes NaN."""
    page = int(tree.page_ids[int(tree.node_page_ptr[node]) + token // 16])
    if tree.mode == "fp8":
        tree.k_pages.view(torch.uint8)[page, head, token % 16, 5] = 0x7F
    else:
        tree.k_pages[page, head, token % 16, 5] = math.nan


def check_with_nans(tree, cap, out, lse, rows, prefill=False, all_nan=False):
    """NaN exactly where 64-bit arithmetic has it (`rows` heads of rows), the rest as near as ever.  (The merge gives
    a row whose sum is NaN lse = -inf, and one whose every score is NaN may pass for one without keys: without a cap
    too.)"""
    ref_o, ref_l, tol_o, tol_l = C.capped(tree, cap, prefill)
    lost = ref_l.isnan()
    assert int(lost.sum()) == rows
    assert (out[lost].isnan() | (all_nan & (out[lost] == 0))).all() and not lse[lost].isfinite().any()
    assert ((out.double() - ref_o).abs() <= tol_o)[~lost].all() and ((lse.double() - ref_l).abs() <= tol_l)[~lost].all()


NAN_CAPS = [(0.0, 1.0), (50.0, 1.0), (10.0, 8.0), (90.0, 1.0), (60.0, 30.0)]


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("heads", [(8, 2), (32, 2)])
@pytest.mark.parametrize("cap,q_std", NAN_CAPS)
def test_nan_stays_in_its_rows(mode, heads, cap, q_std):
    """A NaN score is no score at the cap: it makes its own row NaN and no other."""
    def tree():
        return W.build_tree("nan", [-1] + [0] * 6, [600, 40, 33, 5, 70, 16, 1], [1, 2, 3, 4, 5, 6],
                            num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=128, mode=mode, seed=11, q_std=q_std,
                            device="cuda", tail_value=math.nan)
    group = heads[0] // heads[1]
    own, shared, query = tree(), tree(), tree()
    nan_key(own, 2, 32, 1)                       # the last key of one branch
    check_with_nans(own, cap, *decode(own, cap), group)
    nan_key(shared, 0, 577, 0)
    check_with_nans(shared, cap, *decode(shared, cap), 6 * group)
    if mode != "fp8":
        query.q[3, 1, 7] = math.nan
        check_with_nans(query, cap, *decode(query, cap), 1, all_nan=True)


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
@pytest.mark.parametrize("cap,q_std", NAN_CAPS)
def test_prefill_nan_stays_in_its_rows(mode, cap, q_std):
    """Of a chunk's NaN key: in the rows that see it."""
    for node, token, rows in ((0, 130, (90 + 30) * 4), (1, 70, (90 - 70) * 4), (2, 0, 30 * 4)):
        tree = W.build_prefill("nanp", [-1, 0, 0], [300, 90, 30], [1, 2], num_q_heads=8, num_kv_heads=2, head_dim=128,
                               mode=mode, seed=12, q_std=q_std, device="cuda", tail_value=math.nan)
        nan_key(tree, node, token, 1)
        with Plan.for_prefill(tree, logit_cap=cap) as plan:
            out, lse = plan.decode_tree(tree)
            plan.check()
        check_with_nans(tree, cap, out, lse, rows, prefill=True)
