"""What a decode or a merge allocates belongs to the stream that it runs on: memory that the current stream has
given up, but not yet read, is not written."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import Plan, lse_merge
from tests import fp4_ref as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("what", ["results", "workspace"])
def test_memory_that_is_still_read(what, handle):
    t = F.tree_of([-1] + [0] * 40, [300] + [50] * 40, list(range(1, 41)), 32, 4, seed=3)
    stream = torch.cuda.Stream()
    with Plan.for_tree(t) as plan:
        want, want_lse = (x.clone() for x in plan.decode_tree(t))
        n = plan.workspace_bytes
        plan._ws = None
        ws = torch.empty(n, dtype=torch.uint8, device="cuda") if what == "results" else None
        given = dict(out=torch.empty_like(want), lse=torch.empty_like(want_lse)) if what == "workspace" else {}
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        # blocks of the sizes that the decode will ask for, read late on the current stream
        sizes = [n] if what == "workspace" else [want.numel() * 2, want_lse.numel() * 4]
        blocks = [torch.full((s,), 7, dtype=torch.uint8, device="cuda") for s in sizes]
        copies = [torch.empty_like(b) for b in blocks]
        torch.cuda.synchronize()
        torch.cuda._sleep(200_000_000)                      # (a tenth of a second)
        for c, b in zip(copies, blocks):
            c.copy_(b)
        del b
        blocks.clear()
        out, lse = plan.decode(t.q, t.k_pages, t.v_pages, workspace=ws, k_scale=t.k_scale, v_scale=t.v_scale,
                               stream=stream.cuda_stream if handle else stream, **given)
        torch.cuda.synchronize()
        plan.check()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert all((c == 7).all() for c in copies)


def test_a_merge():
    o, lse = torch.ones((64, 8, 128), device="cuda"), torch.ones((64, 8), device="cuda")
    stream = torch.cuda.Stream()
    want, want_lse = (x.clone() for x in lse_merge(o, lse, o, lse))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    blocks = [torch.full((x.numel() * 4,), 7, dtype=torch.uint8, device="cuda") for x in (want, want_lse)]
    copies = [torch.empty_like(b) for b in blocks]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    for c, b in zip(copies, blocks):
        c.copy_(b)
    del b
    blocks.clear()
    out, out_lse = lse_merge(o, lse, o, lse, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(out_lse, want_lse)
    assert all((c == 7).all() for c in copies)
