"""The scales of an e4m3 or 4-bit decode: contiguous, on the pools' device, or refused."""
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


def trees():
    shape = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, seed=3, device="cuda")
    yield F.tree_of([-1, 0, 0], [70, 33, 5], [1, 2], 8, 2, seed=3)
    yield W.build_tree("scales", [-1, 0, 0], [70, 33, 5], [1, 2], mode="fp8", **shape)


@pytest.mark.parametrize("without", ["decode", "decode_no_alloc"])
def test_scales(without):
    for t in trees():
        with Plan.for_tree(t) as plan:
            def run(ks, vs):
                if without == "decode":
                    return plan.decode(t.q, t.k_pages, t.v_pages, k_scale=ks, v_scale=vs)[0]
                out = torch.empty_like(t.q)
                return plan.decode_no_alloc(t.q, t.k_pages, t.v_pages, out, k_scale=ks, v_scale=vs)[0]
            want = run(t.k_scale, t.v_scale)
            for good in (t.k_scale.view(2, 1), t.k_scale.view(1, 2)):
                assert torch.equal(run(good, t.v_scale), want)
            apart = torch.zeros((2, 3), device="cuda")               # (a layer's column of a table of scales)
            apart[:, 1] = t.k_scale
            one = torch.full((1,), 0.5, device="cuda").expand(2)
            for bad in (apart[:, 1], one, t.k_scale.cpu(), t.k_scale.bfloat16(), t.k_scale[:1]):
                with pytest.raises(ValueError):
                    run(bad, t.v_scale)
                with pytest.raises(ValueError):
                    run(t.k_scale, bad)
            plan.check()
