"""What an e4m3 cache holds is the fp32 quotient with the scale, rounded: to the
bit wherever no rotation goes before."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import kv_write
from tests import kv_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def held(rows, scale):
    """Codes of the quotients, computed on the CPU."""
    x = rows.float().cpu() / scale.cpu().view(-1, 1)
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8).cuda()


def check(k, v, ks, vs, untouched=0, **kw):
    """K from element `untouched` on, and V, to the bit (NaN by its kind)."""
    tokens, heads = k.shape[:2]
    pools = R.pool(R.generator(1), -(-tokens // R.PAGE), heads, 128, "fp8")
    slots = torch.arange(tokens, dtype=torch.int32, device="cuda")
    kv_write(k, v, *pools, slots, k_scale=ks, v_scale=vs, **kw)
    for pool, rows, scale, e in ((pools[0], k, ks, untouched), (pools[1], v, vs, 0)):
        got, want = R.at(pool, slots)[..., e:], held(rows, scale)[..., e:]
        nan = rows[..., e:].isnan()
        assert ((got[nan] & 0x7F) == 0x7F).all()
        assert torch.equal(got[~nan], want[~nan]), f"{int((got != want)[~nan].sum())} codes differ"


@pytest.mark.parametrize("share", [1.0, 0.9])
@pytest.mark.parametrize("kind", [None, (16, 1, False), (64, 1, True)])
def test_scales_from_the_largest_value(share, kind):
    """bf16 values over amax / 448 lie on the ties of e4m3 by the hundred: amax = 7 n / 2^m puts every value that is
    a multiple of n there."""
    gen = R.generator(2)
    for _ in range(4):
        k, v = (torch.randn((500, 16, 128), generator=gen, device="cuda") for _ in range(2))
        k, v = ((x * torch.exp(0.5 * torch.randn((16, 1), generator=gen, device="cuda"))).bfloat16() for x in (k, v))
        ks, vs = (x.float().abs().amax(dim=(0, 2)) * share / 448.0 for x in (k, v))
        rotary, _ = R.rotary_of(kind)
        kw = dict(rotary=rotary, positions=torch.arange(500, dtype=torch.int32, device="cuda")) if kind else {}
        check(k, v, ks, vs, kind[0] if kind else 0, **kw)


def test_every_bf16_value():
    """All 65536 of them over scales from the least the library sets up to 2^126."""
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    rows = every.view(512, 1, 128).expand(512, 16, 128).contiguous()
    gen = R.generator(3)
    scale = torch.exp2(torch.linspace(-92, 126, 16, device="cuda")) * (
        1 + torch.rand(16, generator=gen, device="cuda")).clamp(max=1.99)
    scale[-1] = 2.0 ** 126
    scale[3:7] = torch.tensor([1.0, 1.0 / 448, 3.0, 0.0078125])
    check(rows, rows, scale, scale.flip(0).contiguous())


def test_scales_at_the_ends():
    """From 2^-126 to the largest: a value is off by its rounding and no more than a last place of the quotient."""
    every = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.bfloat16)
    rows = every.view(512, 1, 128).expand(512, 4, 128).contiguous()
    scale = torch.tensor([2.0 ** -126, 2.0 ** -110 * 1.7, 2.0 ** 127, 3.4e38], device="cuda")
    pools = R.pool(R.generator(1), 32, 4, 128, "fp8")
    slots = torch.arange(512, dtype=torch.int32, device="cuda")
    kv_write(rows, rows, *pools, slots, k_scale=scale, v_scale=scale)
    nan = rows.isnan()
    ref = (rows.double() / scale.double().view(-1, 1)).clamp(-448.0, 448.0)
    for pool in pools:
        got = R.at(pool, slots).view(torch.float8_e4m3fn).float().double()
        assert torch.equal(got.isnan(), nan)
        assert ((got - ref).abs() <= R.bound(ref, 0 * ref, torch.float8_e4m3fn, 2))[~nan].all()
