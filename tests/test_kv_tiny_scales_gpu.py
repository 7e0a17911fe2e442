"""K scales of keys so small that the squares of a pair leave fp32."""
import math

import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import Rotary, kv_scales, kv_write
from tests import kv_ref as R
from tests.test_kv_gpu import close, scales_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


@pytest.mark.parametrize("kind", [(128, 1, False), (32, 1, False), (48, 1, True)])
@pytest.mark.parametrize("power", [-40, -50, -55, -60, -64, -70, -74, -80, -100, -115, -120, -130])
def test_norms_of_tiny_pairs(kind, power):
    """A pair's norm, not its larger element, down to where the least scale takes over."""
    gen = R.generator(-power)
    k, v = (R.rows(gen, 70, 5, 128, torch.bfloat16) for _ in range(2))
    k, v = ((x.double() * 2.0 ** power).bfloat16() for x in (k, v))
    k[:, 1] = 0.0                                    # a head of zeros
    k[3, 2] = 1.0                                    # one token of usual size: it decides
    k[:, 3, 1:] = 0.0                                # a partner of zeros
    rotary, _ = R.rotary_of(kind)
    keep = torch.ones(70, dtype=torch.bool, device="cuda")
    got = kv_scales(k, v, rotary=rotary)
    for g, r in zip(got, scales_ref(k, v, rotary, keep)):
        assert close(g, r), (g / r).tolist()


@pytest.mark.parametrize("interleaved", [False, True])
def test_tiny_keys_do_not_saturate(interleaved):
    """Equal elements turned by 45 degrees meet in one of them, at sqrt(2) times their size."""
    freq = torch.zeros(64, device="cuda")
    freq[0] = -math.pi / 4
    rotary = Rotary(freq, interleaved=interleaved)
    k = torch.zeros((16, 1, 128), dtype=torch.bfloat16, device="cuda")
    k[..., 0] = k[..., 1 if interleaved else 64] = 2.0 ** -80
    ks, vs = kv_scales(k, k, rotary=rotary)
    pools = R.pool(R.generator(1), 1, 1, 128, "fp8")
    slots = torch.arange(16, dtype=torch.int32, device="cuda")
    kv_write(k, k, *pools, slots, rotary=rotary, positions=torch.ones(16, dtype=torch.int32, device="cuda"),
             k_scale=ks, v_scale=vs)
    got = R.at(pools[0], slots).view(torch.float8_e4m3fn).float().double() * ks.double()
    # (half a step of e4m3, and what fp32 arithmetic before it adds)
    assert ((got[..., 0] - 2.0 ** -79.5).abs() <= (2.0 ** -4 + 2.0 ** -20) * 2.0 ** -79.5).all()
