"""A capped decode gives the same bits call after call: which form of the tanh a tile takes depends on
its own keys, not on what the warp worked on before."""
import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan
from tests import fp4_ref as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


@pytest.mark.parametrize("mode,d", [("fp4", 128), ("fp8", 128), ("bf16", 128), ("bf16", 64)])
@pytest.mark.parametrize("h_q", [32, 96])
@pytest.mark.parametrize("cap", [5.0, 50.0])
def test_repeats(mode, d, h_q, cap):
    """Branches with logits near the cap and with small ones, in pieces that the warps share out as they
    come: 40 calls, some behind other work."""
    rng = np.random.default_rng(1)
    leaves = 24
    lens = [700] + [int(x) for x in rng.integers(100, 3000, leaves)]
    tree = ([-1] + [0] * leaves, lens, list(range(1, leaves + 1)))
    if mode == "fp4":
        t = F.tree_of(*tree, h_q, 8, seed=2)
    else:
        t = W.build_tree("repeats", *tree, num_q_heads=h_q, num_kv_heads=8, head_dim=d, mode=mode, seed=2, device="cuda")
    size = torch.where(torch.arange(leaves, device="cuda") % 2 == 0, 0.3, 20.0).view(-1, 1, 1)
    t.q.mul_(size.to(t.q.dtype))
    other = torch.empty(1 << 26, device="cuda")
    with Plan.for_tree(t, logit_cap=cap) as plan:
        out, lse = (x.clone() for x in plan.decode_tree(t))
        differ = 0
        for i in range(40):
            if i % 3 == 1:
                other.zero_()
            o, z = plan.decode_tree(t)
            differ += not (torch.equal(o, out) and torch.equal(z, lse))
        plan.check()
    assert differ == 0
