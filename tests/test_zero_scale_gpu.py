"""A kv head whose K scale is 0 (keys of zeros), or so small that its product with the softmax
scale is: every key has the same weight, whatever tile the rows are in."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan
from tests import cap_ref as C
from tests import fp4_ref as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


# (parent, lengths, leaves, heads, prefill): tiles of 4 and 12 rows, a shared prefix's, a prefill's
CASES = {"few": ([-1, 0, 0, 1], [70, 33, 5, 100], [2, 3], (8, 2), False),
         "sixteen": ([-1, 0, 0, 1], [70, 33, 5, 100], [2, 3], (24, 2), False),
         "shared": ([-1] + [0] * 12, [201] + list(range(5, 17)), list(range(1, 13)), (16, 2), False),
         "prefill": ([-1, 0, 0], [77, 40, 130], [1, 2], (8, 2), True)}


@pytest.mark.parametrize("k_scale", [0.0, 2.0 ** -149, 2.0 ** -126])
@pytest.mark.parametrize("cap", [0.0, 50.0, 90.0])
@pytest.mark.parametrize("mode", ["fp4", "fp8"])
@pytest.mark.parametrize("case", sorted(CASES))
def test_k_scale(case, mode, cap, k_scale):
    parent, lens, leaves, (h_q, h_kv), prefill = CASES[case]
    if mode == "fp4":
        t = F.tree_of(parent, lens, leaves, h_q, h_kv, seed=3, prefill=prefill)
    elif prefill:
        t = W.build_prefill("zero", parent, lens, leaves, num_q_heads=h_q, num_kv_heads=h_kv, head_dim=128, mode=mode,
                            seed=3, device="cuda", tail_value=float("nan"))
    else:
        t = W.build_tree("zero", parent, lens, leaves, num_q_heads=h_q, num_kv_heads=h_kv, head_dim=128, mode=mode,
                         seed=3, device="cuda", tail_value=float("nan"))
    t.k_scale[1] = k_scale
    with Plan.for_tree(t, prefill=prefill, logit_cap=cap) as plan:
        out, lse = plan.decode_tree(t)
        plan.check()
    (F if mode == "fp4" else C).check(*((t, out, lse, prefill, cap) if mode == "fp4" else (t, cap, out, lse, prefill)))


@pytest.mark.parametrize("mode", ["fp4", "fp8"])
def test_a_nan_scale_is_a_nan(mode):
    """NaN instead of 0: the head's rows are NaN, the others are not."""
    parent, lens, leaves, (h_q, h_kv), _ = CASES["few"]
    t = (F.tree_of(parent, lens, leaves, h_q, h_kv, seed=4) if mode == "fp4" else
         W.build_tree("nan", parent, lens, leaves, num_q_heads=h_q, num_kv_heads=h_kv, head_dim=128, mode=mode, seed=4,
                      device="cuda"))
    t.k_scale[1] = float("nan")
    with Plan.for_tree(t) as plan:
        out, lse = plan.decode_tree(t)
        plan.check()
    assert torch.isnan(out[:, 4:]).all() and torch.isnan(lse[:, 4:]).all()
    assert torch.isfinite(out[:, :4]).all() and torch.isfinite(lse[:, :4]).all()
