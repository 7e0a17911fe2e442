"""A 4-bit cache written, read and scaled: the bytes against the definition in fp32
where nothing turns, and bounds of a step where fp32 sines and norms come before."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import HeadNorm, Rotary, kv_read, kv_scales, kv_write
from tests import fp4_ref as F
from tests import kv_ref as R
from tests import norm_ref as N

pytestmark = pytest.mark.gpu
D = F.D


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def packed(x, scale):
    """(codes [..., d], scales [..., d / 16]) of x [..., d] in fp32, step by step as defined."""
    b = x.unflatten(-1, (-1, 16))
    most = b.abs().amax(dim=-1)                                        # (NaN stays)
    u = most * (1.0 / (6.0 * scale))
    s = torch.where(torch.isnan(u), u, u.clamp(max=448.0)).to(torch.float8_e4m3fn)
    step = s.float() * scale
    y = b * torch.where(step > 0, 1.0 / step, torch.zeros_like(step)).unsqueeze(-1)
    a = y.abs()
    c = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return (c + 8 * torch.signbit(y).int()).flatten(-2), s.view(torch.uint8)


def bytes_at(pool, slots):
    """(codes [T, H, d], scales [T, H, d / 16]) of the slots."""
    v, s = (x[slots // 16, :, slots % 16] for x in F.split(pool))
    return torch.stack([v & 15, v >> 4], dim=-1).flatten(-2).int(), s


def some_slots(gen, tokens, pages):
    slots = torch.randperm(16 * pages, generator=gen, device="cuda")[:tokens].int()
    if tokens > 2:
        slots[1], slots[tokens - 1] = -1, 16 * pages + 5
    return slots


def check_bytes(pool, before, rows, scale, slots):
    live = (slots >= 0) & (slots < 16 * pool.shape[0])
    at = slots[live].long()
    codes, s = bytes_at(pool, at)
    want, ws = packed(rows[live].float(), scale.view(-1, 1))
    assert torch.equal(s, ws)
    same = codes == want
    same |= (ws == F.NAN_SCALE).repeat_interleave(16, dim=-1)          # (whatever the codes of a NaN block)
    assert same.all()
    rest = torch.ones(16 * pool.shape[0], dtype=torch.bool, device="cuda")
    rest[at] = False
    rest = rest.nonzero().flatten()
    for a, b in zip(F.split(pool), F.split(before)):
        assert torch.equal(a[rest // 16, :, rest % 16], b[rest // 16, :, rest % 16])


@pytest.mark.parametrize("tokens", [1, 2, 37, 700])
@pytest.mark.parametrize("heads,pad,heads_first", [(1, 0, False), (2, 8, False), (5, 0, True), (8, 24, False)])
def test_written_bytes(tokens, heads, pad, heads_first):
    gen = R.generator(tokens + heads)
    pages = tokens // 16 + 2
    k, v = (R.rows(gen, tokens, heads, D, torch.bfloat16, pad, heads_first) for _ in range(2))
    pools = [F.random_pool(gen, pages, heads, 0, 255) for _ in range(2)]
    before = [p.clone() for p in pools]
    slots = some_slots(gen, tokens, pages)
    scales = [0.0005 + 0.002 * torch.rand(heads, generator=gen, device="cuda") for _ in range(2)]
    assert kv_write(k, v, *pools, slots, k_scale=scales[0], v_scale=scales[1]) is None
    for args in zip(pools, before, (k, v), scales):
        check_bytes(*args, slots)


@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-20, 3e-5, 1.0, 7e9, 2.0 ** 100])
def test_values_at_the_ends(scale):
    """Zeros, blocks too small for a scale, saturated ones, ties, infinities, NaN."""
    gen = R.generator(5)
    x = torch.randn((64, 2, D), generator=gen, device="cuda").double()
    x *= 10.0 ** torch.randint(-6, 7, (64, 2, 1), generator=gen, device="cuda")
    x[0] = 0.0
    x[1] = -0.0
    x[2, :, ::2] = 0.0
    x[3] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], device="cuda", dtype=torch.float64).repeat(16)
    x[4] = -x[3]
    x[5] = 2.0 ** -10 * x[3]
    x = (x * scale).to(torch.bfloat16)
    x[6, 0, 17] = float("inf")
    x[7, 1, 40] = float("-inf")
    x[8, 0, 3] = float("nan")
    x[9, 1, 127], x[9, 1, 126] = float("nan"), float("inf")
    pools = [F.random_pool(gen, 4, 2, 0, 255) for _ in range(2)]
    before = [p.clone() for p in pools]
    slots = torch.randperm(64, generator=gen, device="cuda").int()
    scales = torch.full((2,), scale, device="cuda")
    kv_write(x, x.flip(0), *pools, slots, k_scale=scales, v_scale=scales)
    check_bytes(pools[0], before[0], x, scales, slots)
    check_bytes(pools[1], before[1], x.flip(0), scales, slots)
    k, _ = kv_read(*pools, slots, k_scale=scales, v_scale=scales)
    bad = torch.isnan(k)
    assert bad[8, 0, :16].all() and bad[9, 1, 112:].all() and bad.sum() == 32


def check_near(got, ref, loose, scale):
    """got [T, H, d] (64 bits) holds ref within half a step of its block: the exact
    scale rounds to e4m3 (half a step 2^-4, or 2^-10), saturated below 448; half a step of
    a value up to 6 is 1.  `loose`: how far fp32 has ref off."""
    b = ref.unflatten(-1, (-1, 16))
    g = scale.double().view(-1, 1)
    most = b.abs().amax(dim=-1)
    s = torch.maximum(most / (6 * g) * (1 + 2.0 ** -4), most / (6 * g) + 2.0 ** -10).clamp(max=448.0)
    step = (s * g).unsqueeze(-1)
    low = (most / (6 * g) * (1 - 2.0 ** -4) - 2.0 ** -10).clamp(min=0.0, max=448.0).unsqueeze(-1) * g.unsqueeze(-1)
    a = b.abs()
    half = torch.where(a < 2 * low, 0.25, torch.where(a < 4 * low, 0.5, 1.0)) * step
    over = (a - 6 * low).clamp(min=0.0)                                # past the largest value
    off = (got - ref).abs().unflatten(-1, (-1, 16))
    assert (off <= torch.maximum(half, over) * (1 + 2.0 ** -20) + loose.unflatten(-1, (-1, 16))).all()


@pytest.mark.parametrize("kind", [None, (128, 1, False), (128, 1, True), (48, 1, False), (16, 2, False),
                                  (64, 3, False), (112, 1, True)])
@pytest.mark.parametrize("normed", [False, True])
def test_write_and_read_rotated(kind, normed):
    gen = R.generator(21)
    tokens, heads, pages = 45, 2, 5
    rotary, table = R.rotary_of(kind)
    q = R.rows(gen, tokens, 6, D, torch.bfloat16)
    k, v = (R.rows(gen, tokens, heads, D, torch.bfloat16, 16) for _ in range(2))
    norm, w = None, None
    if normed:
        w = [N.weight(gen, (D,), torch.bfloat16) for _ in range(2)]
        norm = HeadNorm(*w)
    pools = [F.random_pool(gen, pages, heads, 0, 255) for _ in range(2)]
    slots = torch.randperm(16 * pages, generator=gen, device="cuda")[:tokens].int()
    positions = None
    if rotary is not None:
        shape = (rotary.num_axes, tokens) if rotary.num_axes > 1 else (tokens,)
        positions = torch.randint(-50, 100000, shape, generator=gen, device="cuda", dtype=torch.int32)
    scales = [0.001 + 0.002 * torch.rand(heads, generator=gen, device="cuda") for _ in range(2)]
    kw = dict(k_scale=scales[0], v_scale=scales[1])
    q_out = kv_write(k, v, *pools, slots, q=q, rotary=rotary, positions=positions, norm=norm, **kw)
    got = kv_read(*pools, slots, **kw)
    for x, weight, out in ((q, w and w[0], q_out), (k, w and w[1], None)):
        ref, size = N.rows(x, weight, rotary, table, positions)
        loose = N.loose(ref, size)
        if out is not None:
            assert ((out.double() - ref).abs() <= loose + R.HALF[torch.bfloat16] * (ref.abs() + loose)).all()
        else:
            held = F.decoded(pools[0], scales[0])[slots.long() // 16, :, slots.long() % 16]
            check_near(held, ref, loose, scales[0])
    held = [F.decoded(p, s)[slots.long() // 16, :, slots.long() % 16] for p, s in zip(pools, scales)]
    check_near(held[1], v.double(), torch.zeros_like(held[1]), scales[1])
    for x, want in zip(got, held):                                     # (a product in fp32, a rounding to bf16)
        assert ((x.double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all()


def test_read_outside_the_pool_and_views():
    gen = R.generator(3)
    pools = [F.random_pool(gen, 3, 4) for _ in range(2)]
    scales = torch.rand(4, generator=gen, device="cuda") + 0.1
    slots = torch.tensor([0, -1, 47, 48, 5, 5, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    buffer = torch.full((8, 2, 4, D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    k, v = kv_read(*pools, slots, k=buffer[:, 0, :, :D], v=buffer[:, 1, :, :D], k_scale=scales, v_scale=scales)
    inside = torch.tensor([0, 2, 4, 5], device="cuda")
    for x, p in ((k, pools[0]), (v, pools[1])):
        want = F.decoded(p, scales)[slots[inside].long() // 16, :, slots[inside].long() % 16]
        assert ((x[inside].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all()
        assert (x[[1, 3, 6, 7]] == 0).all()
    assert (buffer[..., D:] == 7.0).all()


@pytest.mark.parametrize("tokens", [0, 1, 5, 300])
def test_scales(tokens):
    gen = R.generator(tokens)
    k, v = (R.rows(gen, tokens, 3, D, torch.bfloat16) for _ in range(2))
    inv = (1e4 ** (-torch.arange(64, dtype=torch.float64) / 64)).float().cuda()
    rotary = Rotary(inv)
    ks, vs = kv_scales(k, v, rotary=rotary, mode="fp4")
    least = 2.0 ** -100
    if tokens == 0:
        assert (ks == least).all() and (vs == least).all()
        return
    pairs = torch.linalg.vector_norm(k.double().unflatten(-1, (2, 64)), dim=-2).amax(dim=(0, 2)) / 2688
    most = v.double().abs().amax(dim=(0, 2)) / 2688
    assert ((ks.double() - pairs).abs() <= 2.0 ** -21 * pairs).all()
    assert ((vs.double() - most).abs() <= 2.0 ** -23 * most).all()
    more, _ = kv_scales(2 * k, v, rotary=rotary, k_scale=ks.clone(), v_scale=vs.clone(), accumulate=True, mode="fp4")
    assert ((more.double() - 2 * pairs).abs() <= 2.0 ** -20 * pairs).all()
    # tokens written with them keep their largest block within a step
    pools = [F.random_pool(gen, tokens // 16 + 1, 3, 0, 255) for _ in range(2)]
    slots = torch.arange(tokens, dtype=torch.int32, device="cuda")
    kv_write(k, v, *pools, slots, k_scale=ks, v_scale=vs)
    held = F.decoded(pools[1], vs)[slots.long() // 16, :, slots.long() % 16]
    check_near(held, v.double(), torch.zeros_like(held), vs)


def test_a_captured_write():
    gen = R.generator(8)
    k, v = (R.rows(gen, 20, 2, D, torch.bfloat16) for _ in range(2))
    pools = [F.random_pool(gen, 4, 2, 0, 255) for _ in range(2)]
    slots = torch.randperm(64, generator=gen, device="cuda")[:20].int()
    scales = torch.full((2,), 0.001, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv_write(k, v, *pools, slots, k_scale=scales, v_scale=scales)
    slots.copy_(torch.randperm(64, generator=gen, device="cuda")[:20])
    k.mul_(3.0)
    scales.mul_(1.5)
    before = [p.clone() for p in pools]
    graph.replay()
    torch.cuda.synchronize()
    check_bytes(pools[0], before[0], k, scales, slots)
    check_bytes(pools[1], before[1], v, scales, slots)
