"""Writes of so many tokens of few heads that tokens share a warp, into 4 bits and, normed, into the
other types: some of a warp's tokens without a slot, some warps not full."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import HeadNorm, kv_write
from tests import fp4_ref as F
from tests import kv_ref as R
from tests import norm_ref as N
from tests import test_fp4_cache_gpu as cache
from tests import test_head_norm_gpu as normed

pytestmark = pytest.mark.gpu
D = F.D


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def slots_with_holes(gen, tokens, pages):
    """Every seventh token, and every one of 40 in a row, has none (or one outside the pool)."""
    slots = torch.randperm(16 * pages, generator=gen, device="cuda")[:tokens].int()
    slots[::7] = -1
    slots[tokens // 2:tokens // 2 + 40] = 16 * pages + 3
    return slots


# (one wave is about 2400 tokens: from there two tokens share a warp, from twice that four)
@pytest.mark.parametrize("tokens", [2, 3, 2501, 3001, 5003, 9001])
@pytest.mark.parametrize("h_q,heads", [(0, 1), (0, 2), (0, 8), (4, 1), (8, 2)])
def test_written_bytes(tokens, h_q, heads):
    """What nothing turns, byte for byte."""
    gen = R.generator(tokens + heads)
    pages = tokens // 16 + 2
    k, v = (R.rows(gen, tokens, heads, D, torch.bfloat16) for _ in range(2))
    q = R.rows(gen, tokens, h_q, D, torch.bfloat16) if h_q else None
    pools = [F.random_pool(gen, pages, heads, 0, 255) for _ in range(2)]
    before = [p.clone() for p in pools]
    slots = slots_with_holes(gen, tokens, pages)
    scales = [0.0005 + 0.002 * torch.rand(heads, generator=gen, device="cuda") for _ in range(2)]
    out = kv_write(k, v, *pools, slots, q=q, k_scale=scales[0], v_scale=scales[1])
    assert (out is None) if q is None else torch.equal(out, q)
    for args in zip(pools, before, (k, v), scales):
        cache.check_bytes(*args, slots)


@pytest.mark.parametrize("tokens", [3001, 9001])
@pytest.mark.parametrize("h_q,heads", [(0, 1), (0, 8), (4, 1), (8, 2)])
@pytest.mark.parametrize("kind", [None, (128, 1, False), (48, 1, False), (112, 1, True)])
@pytest.mark.parametrize("weights", ["none", "one", "per_head"])
def test_rotated_and_normed(tokens, h_q, heads, kind, weights):
    gen = R.generator(31)
    pages = tokens // 16 + 2
    rotary, table = R.rotary_of(kind)
    q = R.rows(gen, tokens, h_q, D, torch.bfloat16) if h_q else None
    k, v = (R.rows(gen, tokens, heads, D, torch.bfloat16, 16) for _ in range(2))
    norm, w = None, [None, None]
    if weights != "none":
        w = [N.weight(gen, (h, D) if weights == "per_head" else (D,), torch.bfloat16) for h in (max(h_q, 1), heads)]
        norm = HeadNorm(w[0] if h_q else None, w[1])
    pools = [F.random_pool(gen, pages, heads, 0, 255) for _ in range(2)]
    before = [p.clone() for p in pools]
    slots = slots_with_holes(gen, tokens, pages)
    positions = None
    if rotary is not None:
        positions = torch.randint(-50, 100000, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    scales = [0.001 + 0.002 * torch.rand(heads, generator=gen, device="cuda") for _ in range(2)]
    out = kv_write(k, v, *pools, slots, q=q, rotary=rotary, positions=positions, norm=norm, k_scale=scales[0],
                   v_scale=scales[1])
    live = (slots >= 0) & (slots < 16 * pages)
    at = slots[live].long()
    if q is not None:
        ref, size = N.rows(q, w[0], rotary, table, positions)
        loose = N.loose(ref, size)
        assert ((out.double() - ref).abs() <= loose + R.HALF[torch.bfloat16] * (ref.abs() + loose)).all()
    ref, size = N.rows(k, w[1], rotary, table, positions)
    cache.check_near(F.decoded(pools[0], scales[0])[at // 16, :, at % 16], ref[live], N.loose(ref, size)[live], scales[0])
    cache.check_bytes(pools[1], before[1], v, scales[1], slots)
    rest = torch.ones(16 * pages, dtype=torch.bool, device="cuda")
    rest[at] = False
    rest = rest.nonzero().flatten()
    for a, b in zip(F.split(pools[0]), F.split(before[0])):
        assert torch.equal(a[rest // 16, :, rest % 16], b[rest // 16, :, rest % 16])


@pytest.mark.parametrize("mode", ["fp8", "fp32"])
@pytest.mark.parametrize("tokens", [3001, 9001])
def test_normed_into_other_types(mode, tokens):
    normed.check(tokens, mode, 2, 1, D, tokens, (128, 1, False), per_head=True)
    normed.check(tokens, mode, 8, 2, D, tokens, (48, 1, False))
