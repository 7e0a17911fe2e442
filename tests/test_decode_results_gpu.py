"""A decode's given results and workspace: what the kernels would write past, or elsewhere, is
refused before anything is launched; larger buffers, and other shapes of the same memory, are taken."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import ParasonError, Plan
from tests import fp4_ref as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def tree(mode):
    if mode == "fp4":
        return F.tree_of([-1, 0, 0], [70, 33, 5], [1, 2], 8, 2, seed=3)
    return W.build_tree("results", [-1, 0, 0], [70, 33, 5], [1, 2], num_q_heads=8, num_kv_heads=2, head_dim=128,
                        mode=mode, seed=3, device="cuda")


@pytest.mark.parametrize("mode", ["fp4", "fp8", "bf16", "fp32"])
def test_refused(mode):
    t = tree(mode)
    dtype = t.q.dtype
    other = torch.float32 if dtype is torch.bfloat16 else torch.bfloat16
    with Plan.for_tree(t) as plan:
        want, want_lse = plan.decode_tree(t)
        full = dict(dtype=dtype, device="cuda")
        for out in (torch.empty((1, 8, 128), **full), torch.empty((2, 8, 64), **full), torch.empty((2, 8, 128), dtype=other,
                                                                                               device="cuda"),
                    torch.empty((8, 2, 128), **full).transpose(0, 1), torch.empty((1, 8, 128), **full).expand(2, 8, 128),
                    torch.empty((2, 8, 128), dtype=dtype), torch.empty((0,), **full)):
            with pytest.raises(ValueError):
                plan.decode_tree(t, out=out)
        for lse in (torch.empty((2, 7), device="cuda"), torch.empty((2, 8), device="cuda", dtype=torch.bfloat16),
                    torch.empty((8, 2), device="cuda").t(), torch.empty(1, device="cuda").expand(2, 8), torch.empty((2, 8))):
            with pytest.raises(ValueError):
                plan.decode_tree(t, lse=lse)
        n = plan.workspace_bytes
        for ws in (torch.empty(n, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(n + 256),
                   torch.empty((n, 2), dtype=torch.uint8, device="cuda")[:, 0]):
            with pytest.raises(ValueError):
                plan.decode_tree(t, workspace=ws)
        with pytest.raises(ParasonError):
            plan.decode_tree(t, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
        # taken: more rows, one row of all, pinned memory, a workspace of another type
        out, lse = torch.full((3, 8, 128), 7.0, **full), torch.full((20,), 7.0, device="cuda")
        ws = torch.empty(n // 4 + 64, dtype=torch.float32, device="cuda")
        plan.decode_tree(t, out=out, lse=lse, workspace=ws)
        assert torch.equal(out[:2], want) and (out[2] == 7).all()
        assert torch.equal(lse[:16].view(2, 8), want_lse) and (lse[16:] == 7).all()
        out, lse = torch.empty((2, 8, 128), dtype=dtype).pin_memory(), torch.empty((2, 8)).pin_memory()
        plan.decode_tree(t, out=out, lse=lse)
        torch.cuda.synchronize()
        assert torch.equal(out, want.cpu()) and torch.equal(lse, want_lse.cpu())
        out = torch.empty((2, 8, 128), **full)
        assert plan.decode_tree(t, out=out, want_lse=False)[1] is None and torch.equal(out, want)
        plan.check()
