"""The range of V that the kernels without a running maximum (bf16 KV, caps up to
50) promise: 2^34 where 2^20 keys are at the cap, 2^-53 where all are at minus it."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan
from tests import cap_ref as C

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def saturate(tree, sign, low, high):
    """Every logit at sign times the cap; V between low and high, a column's values of one sign (their sum then
    has the size of its terms)."""
    tree.q.fill_(8.0)
    tree.k_pages.fill_(16.0 * sign)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    share = torch.rand(tree.v_pages.shape, generator=gen, device="cuda")
    side = torch.where(torch.arange(tree.head_dim, device="cuda") % 3 == 0, -1.0, 1.0)
    tree.v_pages.copy_(((low + (high - low) * share) * side).bfloat16())
    return tree


def check(tree, out, lse, prefill=False):
    """Equal weights: a row is off by P's rounding and its own (half a step of bf16 each) and the sums of n terms,
    n / 8 + 20 fp32 roundings for each of the two; lse by 2^-18 of 50 (the logit and the sum)."""
    ref_o, ref_l, _, _ = C.capped(tree, 50.0, prefill)
    n = int(tree.node_len.sum())
    assert ((out.double() - ref_o).abs() <= (2.0 ** -7 + 2.0 ** -12 + (n / 4 + 40) * 2.0 ** -24) * ref_o.abs()).all()
    assert ((lse.double() - ref_l).abs() <= 2.0 ** -18 * 50 + (n / 8 + 20) * 2.0 ** -24).all()


ENDS = [(1.0, 2.0 ** 33, 2.0 ** 34), (-1.0, 2.0 ** -53, 2.0 ** -52)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(8, 2), (32, 2)])
@pytest.mark.parametrize("sign,low,high", ENDS)
def test_decode(d, heads, sign, low, high):
    """Suffix steps of both kinds, single tiles and pairs of tiles."""
    tree = saturate(W.build_tree("range", [-1] + [0] * 9, [3000] + [40, 16, 1, 100, 33, 7, 64, 65, 15],
                                 list(range(1, 10)), num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=d, seed=1,
                                 device="cuda"), sign, low, high)
    with Plan.for_tree(tree, logit_cap=50.0) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    check(tree, out, lse)


@pytest.mark.parametrize("sign,low,high", ENDS)
def test_pairs_of_tiles(sign, low, high):
    tree = saturate(W.pair_fixture(mode="bf16", device="cuda"), sign, low, high)
    with Plan.for_tree(tree, logit_cap=50.0) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    check(tree, out, lse)


@pytest.mark.parametrize("sign,low,high", ENDS)
def test_prefill(sign, low, high):
    tree = saturate(W.build_prefill("range", [-1, 0, 0], [900, 90, 30], [1, 2], num_q_heads=8, num_kv_heads=2,
                                    head_dim=128, seed=2, device="cuda"), sign, low, high)
    with Plan.for_prefill(tree, logit_cap=50.0) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    check(tree, out, lse, prefill=True)


def test_a_million_keys_at_the_cap():
    """2^20 keys: out is their mean of V, lse = ln 2^20 + the cap, to the bound's last binade."""
    tree = saturate(W.build_tree("long", [-1, 0, 0], [2 ** 20 - 16, 16, 16], [1, 2], num_q_heads=16, num_kv_heads=1,
                                 head_dim=128, seed=3, device="cuda"), 1.0, 2.0 ** 33, 2.0 ** 34)
    with Plan.for_tree(tree, logit_cap=50.0) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    check(tree, out, lse)
