"""HeadNorm and tensors whose memory is replaced behind it (Tensor.data, as modules do when they
are moved or loaded)."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import HeadNorm, kv_write
from tests import kv_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def inputs(dtype=torch.bfloat16):
    gen = R.generator(1)
    q, k, v = (R.rows(gen, 9, h, 128, dtype) for h in (8, 2, 2))
    mode = "bf16" if dtype is torch.bfloat16 else "fp32"
    return q, k, v, R.pool(gen, 1, 2, 128, mode), torch.arange(9, dtype=torch.int32, device="cuda")


def written(q, k, v, pools, slots, norm):
    pools = [p.clone() for p in pools]
    return [x.view(torch.uint8) for x in (kv_write(k, v, *pools, slots, q=q, norm=norm), *pools)]    # (NaN too)


@pytest.mark.parametrize("shapes", [((128,), (128,)), ((8, 128), (2, 128)), ((128,), (2, 128))])
def test_replaced_weights(shapes):
    """The weights of a write are what the tensors hold then, wherever that lies."""
    gen = R.generator(2)
    args = inputs()

    def make():
        return [torch.nn.Parameter((1 + 0.3 * torch.randn(s, generator=gen, device="cuda")).bfloat16(), False)
                for s in shapes]
    weights, others = make(), make()
    first = [w.data for w in weights]                     # (stays allocated)
    norm = HeadNorm(*weights)
    before = written(*args, norm)
    assert all(torch.equal(a, b) for a, b in zip(before, written(*args, HeadNorm(*first))))
    weights[0].data = others[0].data
    weights[1].data = others[1].data
    after = written(*args, norm)
    assert all(torch.equal(a, b) for a, b in zip(after, written(*args, HeadNorm(*others))))
    assert not torch.equal(before[0], after[0]) and not torch.equal(before[1], after[1])


def test_replaced_by_another_kind():
    """Another type makes the norm one for rows of it; weights that no norm takes are refused at the write."""
    args = inputs()
    weights = [torch.nn.Parameter(torch.full((128,), 1.5, device="cuda", dtype=torch.bfloat16), False) for _ in range(2)]
    kept = [w.data for w in weights]                      # (stays allocated)
    norm = HeadNorm(*weights)
    for w in weights:
        w.data = w.data.float()
    with pytest.raises(ValueError):
        written(*args, norm)
    wide = inputs(torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(written(*wide, norm), written(*wide, HeadNorm(*(w.float() for w in kept)))))
    for bad in (torch.ones(64, device="cuda", dtype=torch.bfloat16), torch.ones((3, 128), device="cuda", dtype=torch.bfloat16),
                torch.ones(128, dtype=torch.bfloat16), torch.ones(256, device="cuda", dtype=torch.bfloat16)[::2],
                torch.ones(136, device="cuda", dtype=torch.bfloat16)[1:129]):
        fresh = [torch.nn.Parameter(x.clone(), False) for x in kept]
        norm, held = HeadNorm(*fresh), [w.data for w in fresh]
        fresh[1].data = bad
        with pytest.raises(ValueError):
            written(*args, norm)
        del held


def test_weights_that_are_given_up():
    """No write without their memory; with new memory the norm goes on."""
    args = inputs()
    w = torch.full((128,), 1.5, device="cuda", dtype=torch.bfloat16)
    norm = HeadNorm(w, w)
    w.untyped_storage().resize_(0)
    with pytest.raises(ValueError):
        written(*args, norm)
    w.untyped_storage().resize_(256)
    w.fill_(0.75)
    want = written(*args, HeadNorm(*(torch.full_like(w, 0.75) for _ in range(2))))
    assert all(torch.equal(a, b) for a, b in zip(written(*args, norm), want))
