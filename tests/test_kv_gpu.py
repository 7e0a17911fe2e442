"""kv_write, kv_read and kv_scales against 64-bit arithmetic, at the sizes,
strides, slots and values where they can go wrong."""
import math

import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import Rotary, kv_read, kv_scales, kv_write
from tests import kv_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def spread_slots(gen, tokens, pages, outside=True):
    """Distinct slots in any order, some tokens without one."""
    slots = torch.randperm(pages * R.PAGE, generator=gen, device="cuda")[:tokens].to(torch.int32)
    if outside and tokens > 2:
        slots[1], slots[tokens - 1] = -1, pages * R.PAGE + 3
    return slots


def positions_for(gen, rotary, tokens, lo=-50, hi=5000):
    if rotary is None:
        return None
    shape = (rotary.num_axes, tokens) if rotary.num_axes > 1 else (tokens,)
    return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)


def check_write(seed, mode, h_q, h_kv, d, tokens, kind, pad=0, heads_first=False, lo=-50, hi=5000):
    gen = R.generator(seed)
    rotary, table = R.rotary_of(kind)
    dtype, pages = R.ROWS[mode], tokens // R.PAGE + 4
    q, k, v = (R.rows(gen, tokens, h, d, dtype, pad, heads_first) for h in (h_q, h_kv, h_kv))
    pools = R.pool(gen, pages, h_kv, d, mode)
    before = [p.clone() for p in pools]
    slots = spread_slots(gen, tokens, pages)
    positions = positions_for(gen, rotary, tokens, lo, hi)
    scales = [0.004 + 0.004 * torch.rand(h_kv, generator=gen, device="cuda") for _ in range(2)]
    q_out = kv_write(k, v, *pools, slots, q=q, rotary=rotary, positions=positions,
                     k_scale=scales[0], v_scale=scales[1])
    ref, size = R.rotated(q, rotary, table, positions)
    assert q_out.is_contiguous() and q_out.shape == q.shape
    assert ((q_out.double() - ref).abs() <= R.bound(ref, size, dtype)).all()
    live = (slots >= 0) & (slots < pages * R.PAGE)
    untouched = torch.ones(pages * R.PAGE, dtype=torch.bool, device="cuda")
    untouched[slots[live].long()] = False
    for pool, old, rows, scale, turned in ((pools[0], before[0], k, scales[0], True),
                                           (pools[1], before[1], v, scales[1], False)):
        ref, size = R.rotated(rows, rotary if turned else None, table, positions)
        if mode == "fp8":
            ref, size = R.stored(ref, size, scale)
        got = R.at(pool, slots[live]).view(pool.dtype).double() if mode != "fp8" else \
            R.at(pool, slots[live]).view(pool.dtype).float().double()
        # (a scale's reciprocal and the product with it round)
        assert ((got - ref[live]).abs() <= R.bound(ref, size, pool.dtype, 2)[live]).all()
        rest = torch.arange(pages * R.PAGE, device="cuda")[untouched]
        assert torch.equal(R.at(pool, rest), R.at(old, rest))


HALVES, PART, MIXED, AXES = (128, 1, False), (32, 1, False), (48, 1, True), (64, 3, False)


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("kind", [None, HALVES, (128, 1, True), PART, MIXED, AXES, (128, 4, True), (16, 2, False)])
def test_write_rotary_kinds(mode, kind):
    check_write(1, mode, 8, 2, 128, 37, kind)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", [None, (64, 1, False), (64, 3, True), (16, 1, True)])
def test_write_head_dim_64(mode, kind):
    check_write(2, mode, 6, 3, 64, 21, kind)


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("tokens", [1, 2, 3, 7, 8, 9, 16, 31, 64, 65, 255, 1000])
def test_write_lengths(mode, tokens):
    check_write(tokens, mode, 4, 1, 128, tokens, HALVES, pad=8)


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
@pytest.mark.parametrize("heads", [(1, 1), (5, 1), (64, 8), (28, 4), (16, 16), (96, 32)])
def test_write_head_layouts(mode, heads):
    check_write(3, mode, *heads, 128, 19, AXES)


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("pad,heads_first", [(8, False), (24, False), (0, True), (16, True)])
def test_write_strides(mode, pad, heads_first):
    check_write(4, mode, 8, 2, 128, 40, HALVES, pad=pad, heads_first=heads_first)


@pytest.mark.parametrize("mode,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64), ("fp8", 128)])
@pytest.mark.parametrize("heads,kind", [((8, 2), MIXED), ((1, 1), AXES), ((5, 1), None), ((12, 3), (16, 4, False))])
@pytest.mark.parametrize("tokens", [4865, 9733])
def test_write_many_tokens_of_few_heads(mode, d, heads, kind, tokens):
    """Two and four tokens share a warp; the last warp lacks some."""
    if kind is not None and kind[0] > d:
        pytest.skip("rotary_dim above head_dim")
    check_write(tokens, mode, *heads, d, tokens, kind, pad=8)


@pytest.mark.parametrize("tokens,heads", [(700, 32), (1217, 16), (2433, 24), (3041, 8)])
def test_write_around_a_wave_of_warps(tokens, heads):
    """Where the parts of a token change in number, and end."""
    check_write(9, "bf16", heads, 8, 128, tokens, HALVES)


@pytest.mark.parametrize("lo,hi", [(2 ** 20, 2 ** 20 + 5000), (-2 ** 24, 2 ** 24)])
def test_write_far_positions(lo, hi):
    """Up to 2^24 the reduced angle is as near as at the origin."""
    check_write(5, "fp32", 4, 2, 128, 100, HALVES, lo=lo, hi=hi)


def test_write_farthest_positions():
    """At the ends of int32 the reference's angle, up to 2^31 radians in 64 bits, is off
    by 2^-22 radians itself; the kernel's is as near as elsewhere."""
    rotary, table = R.rotary_of(HALVES)
    gen = R.generator(6)
    positions = torch.tensor([2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 0], dtype=torch.int32, device="cuda")
    q, k = (R.rows(gen, 4, h, 128, torch.float32) for h in (2, 1))
    pools = R.pool(gen, 1, 1, 128, "fp32")
    out = kv_write(k, k, *pools, torch.full((4,), -1, dtype=torch.int32, device="cuda"), q=q, rotary=rotary,
                   positions=positions)
    ref, size = R.rotated(q, rotary, table, positions)
    assert ((out.double() - ref).abs() <= R.bound(ref, size, torch.float32) + 2.0 ** -22 * size).all()


def test_write_special_values():
    """Infinities saturate, NaN stays, zeros and the largest values keep their sign."""
    scale = torch.tensor([0.5], device="cuda")
    x = torch.zeros((4, 1, 128), dtype=torch.bfloat16, device="cuda")
    x[0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, -0.0])
    x[1, 0, :4] = torch.tensor([224.0, -224.0, 3e38, -3e38])
    x[2, 0, :3] = torch.tensor([2.0 ** -11, 2.0 ** -12, 1e-38])       # half of the least step: to even, 0
    pools = R.pool(R.generator(7), 1, 1, 128, "fp8")
    slots = torch.tensor([3, 0, 15, 7], dtype=torch.int32, device="cuda")
    kv_write(x, x, *pools, slots, k_scale=scale, v_scale=scale)
    for pool in pools:
        got = R.at(pool, slots).view(pool.dtype).float()
        assert got[0, 0, 0] == 448 and got[0, 0, 1] == -448 and got[0, 0, 2].isnan() and got[0, 0, 3] == 0
        assert got[1, 0, :4].tolist() == [448, -448, 448, -448]
        assert got[2, 0, :3].tolist() == [0, 0, 0] and (got[:, 0, 4:] == 0).all()
    # rotated NaN and infinities stay in their own pairs
    rotary, _ = R.rotary_of(HALVES)
    bf = R.pool(R.generator(8), 1, 1, 128, "bf16")
    out = kv_write(x, x, *bf, slots, q=x, rotary=rotary,
                   positions=torch.arange(5, 9, dtype=torch.int32, device="cuda"))
    bad = ~out[0, 0].isfinite()
    assert bad[[0, 1, 2, 64, 65, 66]].all() and bad.sum() == 6


def test_write_without_and_with_q_in_place():
    gen = R.generator(9)
    rotary, table = R.rotary_of(HALVES)
    positions = torch.arange(33, dtype=torch.int32, device="cuda")
    k, v = (R.rows(gen, 33, 2, 128, torch.bfloat16) for _ in range(2))
    q = R.rows(gen, 33, 8, 128, torch.bfloat16)
    slots = spread_slots(gen, 33, 5)
    pools, again = R.pool(gen, 5, 2, 128, "bf16"), None
    assert kv_write(k, v, *pools, slots, rotary=rotary, positions=positions) is None
    again = [p.clone() for p in pools]
    ref, size = R.rotated(q, rotary, table, positions)
    assert kv_write(k, v, *pools, slots, q=q, q_out=q, rotary=rotary, positions=positions) is q
    assert ((q.double() - ref).abs() <= R.bound(ref, size, torch.bfloat16)).all()
    assert all(torch.equal(R.raw(a), R.raw(b)) for a, b in zip(pools, again))


def test_empty_batch_and_empty_pool():
    k = torch.empty((0, 2, 128), dtype=torch.bfloat16, device="cuda")
    pools = R.pool(R.generator(10), 2, 2, 128, "bf16")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    old = [p.clone() for p in pools]
    out = kv_write(k, k, *pools, none, q=torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda"))
    assert out.shape == (0, 4, 128)
    assert all(t.shape == (0, 2, 128) for t in kv_read(*pools, none))
    assert all(torch.equal(R.raw(a), R.raw(b)) for a, b in zip(pools, old))
    ks, vs = kv_scales(k, k)
    assert (ks == 2.0 ** -126).all() and (vs == 2.0 ** -126).all()
    empty = [p[:0] for p in pools]
    x = torch.ones((3, 2, 128), dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([0, -1, 5], dtype=torch.int32, device="cuda")
    assert torch.equal(kv_write(x, x, *empty, slots, q=x), x)
    assert all((t == 0).all() for t in kv_read(*empty, slots))


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("kind", [HALVES, AXES])
def test_empty_batch_with_positions(mode, kind):
    rotary, _ = R.rotary_of(kind)
    k = torch.empty((0, 2, 128), dtype=R.ROWS[mode], device="cuda")
    pools = R.pool(R.generator(10), 2, 2, 128, mode)
    one = torch.ones(2, device="cuda")
    shape = (0,) if rotary.num_axes == 1 else (rotary.num_axes, 0)
    out = kv_write(k, k, *pools, torch.empty(0, dtype=torch.int32, device="cuda"), q=k, rotary=rotary,
                   positions=torch.empty(shape, dtype=torch.int32, device="cuda"), k_scale=one, v_scale=one)
    assert out.shape == (0, 2, 128)


@pytest.mark.parametrize("mode,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64), ("fp8", 128)])
@pytest.mark.parametrize("tokens", [1, 2, 15, 64, 129, 1000])
def test_read(mode, d, tokens):
    gen = R.generator(tokens)
    pools = [x.to(R.POOL[mode]) for x in torch.randn((2, 9, 3, R.PAGE, d), generator=gen, device="cuda")]
    scales = [torch.rand(3, generator=gen, device="cuda") + 0.1 for _ in range(2)]
    slots = torch.randint(-2, 9 * R.PAGE + 2, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    got = kv_read(*pools, slots, k_scale=scales[0], v_scale=scales[1])
    live = (slots >= 0) & (slots < 9 * R.PAGE)
    for pool, scale, rows in zip(pools, scales, got):
        assert rows.dtype == R.ROWS[mode] and rows.is_contiguous()
        ref = R.at(pool, slots[live]).view(pool.dtype).float().double()
        if mode == "fp8":
            ref = ref * scale.double().view(-1, 1)
            assert ((rows[live].double() - ref).abs() <= R.bound(ref, 0 * ref, torch.bfloat16)).all()
        else:
            assert torch.equal(rows[live].double(), ref)
        assert (rows[~live] == 0).all()


@pytest.mark.parametrize("mode,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64), ("fp8", 128)])
@pytest.mark.parametrize("heads", [1, 2, 5, 17, 33, 300])
@pytest.mark.parametrize("tokens", [1, 3, 131])
def test_read_head_counts(mode, d, heads, tokens):
    """A warp's rows begin at any head, end in another token, and pass several."""
    gen = R.generator(heads)
    pools = [x.to(R.POOL[mode]) for x in torch.randn((2, 5, heads, R.PAGE, d), generator=gen, device="cuda")]
    scales = [torch.full((heads,), 1.0, device="cuda") * 2.0 ** torch.randint(-3, 4, (heads,), generator=gen,
                                                                             device="cuda") for _ in range(2)]
    slots = torch.randint(-1, 5 * R.PAGE + 1, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    live = (slots >= 0) & (slots < 5 * R.PAGE)
    got = kv_read(*pools, slots, k_scale=scales[0], v_scale=scales[1])
    for pool, scale, rows in zip(pools, scales, got):
        ref = R.at(pool, slots[live]).view(pool.dtype).float()
        if mode == "fp8":
            ref = ref * scale.view(-1, 1)            # (a power of 2: the product is exact in bf16)
        assert torch.equal(rows[live].float(), ref) and (rows[~live] == 0).all()


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
def test_read_into_views(mode):
    """Rows into a wider buffer; what lies between them stays."""
    gen = R.generator(11)
    pools = [x.to(R.POOL[mode]) for x in torch.randn((2, 4, 2, R.PAGE, 128), generator=gen, device="cuda")]
    one = torch.ones(2, device="cuda")
    wide = torch.full((20, 2, 2, 136), 7.0, dtype=R.ROWS[mode], device="cuda")
    k, v = wide[:, 0, :, :128], wide[:, 1, :, :128]
    slots = torch.randint(0, 64, (20,), generator=gen, device="cuda", dtype=torch.int32)
    got = kv_read(*pools, slots, k=k, v=v, k_scale=one, v_scale=one)
    assert got[0] is k and got[1] is v and (wide[..., 128:] == 7).all()
    for pool, rows in zip(pools, got):
        assert torch.equal(rows.float(), R.at(pool, slots).view(pool.dtype).float())


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
def test_read_into_heads_first(mode):
    gen = R.generator(12)
    pools = [x.to(R.POOL[mode]) for x in torch.randn((2, 4, 2, R.PAGE, 128), generator=gen, device="cuda")]
    one = torch.ones(2, device="cuda")
    slots = torch.randint(0, 64, (20,), generator=gen, device="cuda", dtype=torch.int32)
    k, v = (torch.empty((2, 20, 136), dtype=R.ROWS[mode], device="cuda")[..., 8:].transpose(0, 1) for _ in range(2))
    kv_read(*pools, slots, k=k, v=v, k_scale=one, v_scale=one)
    for pool, rows in zip(pools, (k, v)):
        assert torch.equal(rows.float(), R.at(pool, slots).view(pool.dtype).float())


def test_read_every_e4m3_code():
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(2, 1, 1, 128).expand(2, 1, R.PAGE, 128)
    pool = codes.contiguous().view(torch.float8_e4m3fn)
    scale = torch.tensor([1.0], device="cuda")
    slots = torch.tensor([0, 16], dtype=torch.int32, device="cuda")
    k, v = kv_read(pool, pool, slots, k_scale=scale, v_scale=scale)
    want = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).float()
    for rows in (k, v):
        got = rows.float().reshape(-1)
        assert torch.equal(got.isnan(), want.isnan())
        assert torch.equal(got[~want.isnan()], want[~want.isnan()])


def scales_ref(k, v, rotary, keep):
    k, v = k[keep].double().abs(), v[keep].double().abs()
    k, v = (x.nan_to_num(0.0).clamp(max=2.0 ** 63) for x in (k, v))
    best = k.amax(dim=(0, 2)) if k.shape[0] else torch.zeros(k.shape[1], dtype=torch.float64, device="cuda")
    if rotary is not None and k.shape[0]:
        r = rotary.rotary_dim
        a, b = ((k[..., 0:r:2], k[..., 1:r:2]) if rotary.interleaved else (k[..., :r // 2], k[..., r // 2:r]))
        best = torch.maximum(best, torch.hypot(a, b).amax(dim=(0, 2)))
    vbest = v.amax(dim=(0, 2)) if v.shape[0] else torch.zeros_like(best)
    return [(x / 448).clamp(min=2.0 ** -126) for x in (best, vbest)]


def close(got, ref):
    """Squares, their sum, the root and the quotient round in fp32: at most 2 + 1 / 2 + 1 steps."""
    return bool(((got.double() - ref).abs() <= 4 * 2.0 ** -24 * ref).all())


@pytest.mark.parametrize("tokens", [1, 2, 33, 256, 257, 5000])
@pytest.mark.parametrize("heads", [1, 2, 8, 17])
@pytest.mark.parametrize("kind", [None, HALVES, MIXED])
def test_scales(tokens, heads, kind):
    gen = R.generator(tokens * 31 + heads)
    k, v = (R.rows(gen, tokens, heads, 128, torch.bfloat16, pad=8) for _ in range(2))
    rotary, _ = R.rotary_of(kind)
    got = kv_scales(k, v, rotary=rotary)
    keep = torch.ones(tokens, dtype=torch.bool, device="cuda")
    assert all(close(g, r) for g, r in zip(got, scales_ref(k, v, rotary, keep)))
    # tokens without a slot do not count
    slots = torch.randint(-3, 4, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    got = kv_scales(k, v, rotary=rotary, slots=slots)
    assert all(close(g, r) for g, r in zip(got, scales_ref(k, v, rotary, slots >= 0)))


def test_scales_of_odd_values():
    k = torch.zeros((3, 4, 128), dtype=torch.bfloat16, device="cuda")
    k[0, 0, 5] = math.nan
    k[1, 1, 7], k[2, 1, 71] = -math.inf, 3.0
    k[0, 2, 1], k[0, 2, 65] = 2.0 ** 62, -2.0 ** 62
    k[2, 3, 100] = 2.0 ** -100
    rotary, _ = R.rotary_of(HALVES)
    keep = torch.ones(3, dtype=torch.bool, device="cuda")
    for rot in (None, rotary):
        got = kv_scales(k, k, rotary=rot)
        assert all(close(g, r) for g, r in zip(got, scales_ref(k, k, rot, keep))), (got, rot)


def test_scales_accumulate_in_any_order():
    gen = R.generator(12)
    rotary, _ = R.rotary_of(HALVES)
    batches = [R.rows(gen, n, 4, 128, torch.bfloat16) for n in (300, 1, 77)]
    whole = kv_scales(torch.cat(batches), torch.cat(batches), rotary=rotary)
    for order in ((0, 1, 2), (2, 0, 1)):
        ks, vs = torch.full((4,), 1e-9, device="cuda"), torch.full((4,), 1e-9, device="cuda")
        for i in order:
            kv_scales(batches[i], batches[i], rotary=rotary, k_scale=ks, v_scale=vs, accumulate=True)
        assert torch.equal(ks, whole[0]) and torch.equal(vs, whole[1])
    ks, vs = torch.full((4,), 5.0, device="cuda"), torch.full((4,), 6.0, device="cuda")
    kv_scales(batches[0], batches[0], k_scale=ks, v_scale=vs, accumulate=True)
    assert (ks == 5).all() and (vs == 6).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_scales_hold_rotated_keys(interleaved):
    """No position takes a key past 448 scales by more than its own rounding."""
    gen = R.generator(13)
    rotary, table = R.rotary_of((128, 1, interleaved))
    k, v = (R.rows(gen, 64, 2, 128, torch.bfloat16) for _ in range(2))
    ks, _ = kv_scales(k, v, rotary=rotary)
    for base in (0, 1000, -77777):
        pos = base + torch.arange(64, dtype=torch.int32, device="cuda")
        turned, _ = R.rotated(k, rotary, table, pos)
        assert (turned.abs().amax(dim=(0, 2)) <= 448 * ks.double() * (1 + 2.0 ** -20)).all()


def test_replay_with_new_slots_and_positions():
    """A captured write and read follow the slots, positions, rows and scales that the buffers hold at replay."""
    gen = R.generator(14)
    rotary, table = R.rotary_of(HALVES)
    k, v = (R.rows(gen, 8, 2, 128, torch.bfloat16) for _ in range(2))
    q = R.rows(gen, 8, 4, 128, torch.bfloat16)
    slots = torch.arange(8, dtype=torch.int32, device="cuda")
    pos = torch.arange(8, dtype=torch.int32, device="cuda")
    ks, vs, q_out = torch.ones(2, device="cuda"), torch.ones(2, device="cuda"), torch.empty_like(q)
    pools = [p.zero_() for p in R.pool(gen, 3, 2, 128, "fp8")]
    back = [torch.empty_like(k) for _ in range(2)]

    def step():
        kv_scales(k, v, rotary=rotary, k_scale=ks, v_scale=vs)
        kv_write(k, v, *pools, slots, q=q, q_out=q_out, rotary=rotary, positions=pos, k_scale=ks, v_scale=vs)
        kv_read(*pools, slots, k=back[0], v=back[1], k_scale=ks, v_scale=vs)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for shift in (0, 11, 29):
        slots.copy_((torch.arange(8, device="cuda") * 5 + shift) % 48)
        pos.copy_(torch.arange(8, device="cuda") + 1000 * shift)
        k.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        ref, size = R.rotated(k, rotary, table, pos)
        got_scale = ks.clone()
        held, held_size = R.stored(ref, size, got_scale)
        stored = R.at(pools[0], slots).view(torch.float8_e4m3fn).float()
        assert ((stored.double() - held).abs() <= R.bound(held, held_size, torch.float8_e4m3fn, 2)).all()
        want = stored.double() * got_scale.double().view(-1, 1)
        assert ((back[0].double() - want).abs() <= R.bound(want, 0 * want, torch.bfloat16)).all()
        ref, size = R.rotated(q, rotary, table, pos)
        assert ((q_out.double() - ref).abs() <= R.bound(ref, size, torch.bfloat16)).all()


@pytest.mark.parametrize("which", ["stream", "handle", "default"])
def test_another_stream(which):
    """New outputs belong to the stream that writes them."""
    gen = R.generator(15)
    k, v = (R.rows(gen, 100, 2, 128, torch.bfloat16) for _ in range(2))
    pools = R.pool(gen, 8, 2, 128, "bf16")
    slots = torch.randperm(128, generator=gen, device="cuda")[:100].to(torch.int32)
    side = torch.cuda.default_stream() if which == "default" else torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    handle = {"stream": side, "handle": side.cuda_stream, "default": 0}[which]
    q = kv_write(k, v, *pools, slots, q=k, stream=handle)
    rk, rv = kv_read(*pools, slots, stream=handle)
    ks, vs = kv_scales(k, v, stream=handle)
    side.synchronize()
    assert torch.equal(q, k) and torch.equal(rk, k) and torch.equal(rv, v)
    assert close(ks, k.double().abs().amax(dim=(0, 2)) / 448)


def test_slots_past_32_bit_offsets():
    """Elements of the last pages lie past 2^31 elements and 2^32 bytes."""
    pages, heads = 2 ** 31 // (8 * R.PAGE * 128) + 40, 8
    pools = [torch.zeros((pages, heads, R.PAGE, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    gen = R.generator(16)
    k, v = (R.rows(gen, 48, heads, 128, torch.bfloat16) for _ in range(2))
    slots = (pages - 3) * R.PAGE + torch.randperm(48, generator=gen, device="cuda").to(torch.int32)
    kv_write(k, v, *pools, slots)
    assert torch.equal(R.at(pools[0], slots), R.raw(k)) and torch.equal(R.at(pools[1], slots), R.raw(v))
    assert int((pools[0][:pages - 3] != 0).sum()) == 0
    rk, rv = kv_read(*pools, slots)
    assert torch.equal(rk, k) and torch.equal(rv, v)


def test_refusals_of_the_binding():
    gen = R.generator(17)
    k = R.rows(gen, 4, 2, 128, torch.bfloat16)
    pools = R.pool(gen, 2, 2, 128, "bf16")
    slots = torch.arange(4, dtype=torch.int32, device="cuda")
    rotary, _ = R.rotary_of(HALVES)
    three, _ = R.rotary_of(AXES)
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    bad = [
        dict(k=k.float()), dict(k=k[:3]), dict(k=k.cpu()), dict(slots=slots.long()), dict(slots=slots[:3]),
        dict(slots=slots.cpu()), dict(rotary=rotary), dict(positions=pos), dict(q_out=k),
        dict(rotary=rotary, positions=pos.long()), dict(rotary=rotary, positions=pos[:3]),
        dict(rotary=three, positions=pos), dict(q=k[:, :1]), dict(q=k, q_out=k[:, :1]),
        dict(q=torch.zeros((4, 2, 130), dtype=torch.bfloat16, device="cuda")[..., :128]),
        dict(v=torch.zeros((4, 2, 256), dtype=torch.bfloat16, device="cuda")[..., ::2]),
        dict(k_pages=pools[0].view(torch.float8_e4m3fn)[..., :128]), dict(v_pages=pools[1][:1]),
        dict(k_pages=pools[0].half(), v_pages=pools[1].half())]
    for change in bad:
        with pytest.raises(ValueError):
            kv_write(**dict(dict(k=k, v=k, k_pages=pools[0], v_pages=pools[1], slots=slots), **change))
    view = torch.zeros((4, 4, 128), dtype=torch.bfloat16, device="cuda")[:, ::2]
    with pytest.raises(ValueError):
        kv_write(k, k, *pools, slots, q=view, q_out=view)
    f8 = [torch.zeros((2, 2, 16, 128), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    one = torch.ones(2, device="cuda")
    for scales in (dict(), dict(k_scale=one), dict(k_scale=one, v_scale=one[:1]),
                   dict(k_scale=one, v_scale=one.double())):
        with pytest.raises(ValueError):
            kv_write(k, k, *f8, slots, **scales)
        with pytest.raises(ValueError):
            kv_read(*f8, slots, **scales)
    with pytest.raises(ValueError):
        kv_read(*pools, slots.view(2, 2))
    with pytest.raises(ValueError):
        kv_read(*pools, slots, k=k[:1].expand(4, 2, 128))
    for strides in ((128, 128, 1), (248, 128, 1), (136, 528, 1), (256, 256, 1)):
        with pytest.raises(ValueError):
            kv_read(*pools, slots, k=torch.zeros(2048, dtype=torch.bfloat16,
                                                 device="cuda").as_strided((4, 2, 128), strides))
    with pytest.raises(ValueError):
        kv_scales(k.float(), k.float())
    with pytest.raises(ValueError):
        kv_scales(k, k, accumulate=True)
    for inv, axes in ((torch.ones(4, device="cuda"), None), (torch.ones(72, device="cuda"), None),
                      (torch.ones(8), None), (torch.ones(8, device="cuda"), [0] * 7),
                      (torch.ones(8, device="cuda"), [4] * 8), (torch.ones(8, device="cuda"), [-1] * 8),
                      (torch.ones(8, device="cuda"), [0.5] * 8)):
        with pytest.raises(ValueError):
            Rotary(inv, axes=axes)
