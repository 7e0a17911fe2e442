"""kv_write with q and k normed head by head, into every type of cache, against 64 bits."""
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import HeadNorm, kv_write
from tests import kv_ref as R
from tests import norm_ref as N

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def check(seed, mode, h_q, h_kv, d, tokens, kind, per_head=False, which="qk", eps=N.EPS, offset=0.0, size=1.0,
          pad=0, heads_first=False):
    gen = R.generator(seed)
    rotary, table = R.rotary_of(kind)
    dtype, pages = R.ROWS[mode], tokens // 16 + 3
    q, k, v = (R.rows(gen, tokens, h, d, dtype, pad, heads_first) for h in (h_q, h_kv, h_kv))
    q.mul_(size), k.mul_(size)
    w = [N.weight(gen, (h, d) if per_head else (d,), dtype, offset) if c in which else None
         for c, h in zip("qk", (h_q, h_kv))]
    norm = HeadNorm(*w, eps=eps, unit_offset=offset == 1.0)
    pools = R.pool(gen, pages, h_kv, d, mode)
    before = [p.clone() for p in pools]
    slots = torch.randperm(16 * pages, generator=gen, device="cuda")[:tokens].int()
    if tokens > 2:
        slots[1] = -1
    positions = None
    if rotary is not None:
        shape = (rotary.num_axes, tokens) if rotary.num_axes > 1 else (tokens,)
        positions = torch.randint(-50, 100000, shape, generator=gen, device="cuda", dtype=torch.int32)
    scales = [0.01 + 0.004 * torch.rand(h_kv, generator=gen, device="cuda") for _ in range(2)]
    q_out = kv_write(k, v, *pools, slots, q=q, rotary=rotary, positions=positions, norm=norm, k_scale=scales[0],
                     v_scale=scales[1])
    ref, pair = N.rows(q, w[0], rotary, table, positions, eps, offset)
    off = N.loose(ref, pair)
    assert ((q_out.double() - ref).abs() <= off + R.HALF[dtype] * (ref.abs() + off) + R.TINY[dtype]).all()
    live = slots >= 0
    untouched = torch.ones(16 * pages, dtype=torch.bool, device="cuda")
    untouched[slots[live].long()] = False
    rest = untouched.nonzero().flatten()
    for pool, old, x, weight, scale, rot in ((pools[0], before[0], k, w[1], scales[0], rotary),
                                             (pools[1], before[1], v, None, scales[1], None)):
        ref, pair = N.rows(x, weight, rot, table, positions, eps, offset)
        off = N.loose(ref, pair)
        if mode == "fp8":
            s = scale.double().view(-1, 1)
            ref, off = (ref / s).clamp(-448.0, 448.0), off / s + 2.0 ** -23 * (ref / s).abs()
        got = R.at(pool, slots[live]).view(pool.dtype)
        got = got.float().double() if mode == "fp8" else got.double()
        most = off + R.HALF[pool.dtype] * (ref.abs() + off) + R.TINY[pool.dtype]
        assert ((got - ref[live]).abs() <= most[live]).all()
        assert torch.equal(R.at(pool, rest), R.at(old, rest))


KINDS = [None, (128, 1, False), (128, 1, True), (32, 1, False), (48, 3, False)]


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
@pytest.mark.parametrize("kind", KINDS)
def test_kinds(mode, kind):
    check(1, mode, 8, 2, 128, 37, kind)


@pytest.mark.parametrize("mode", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", [None, (64, 1, False), (16, 1, True)])
def test_head_dim_64(mode, kind):
    check(2, mode, 6, 3, 64, 21, kind)


@pytest.mark.parametrize("tokens", [1, 2, 16, 500, 6000])
@pytest.mark.parametrize("heads", [(5, 1), (32, 8), (16, 16)])
def test_counts(tokens, heads):
    check(tokens, "bf16", *heads, 128, tokens, (128, 1, False))


@pytest.mark.parametrize("tokens", [3, 9000])
def test_tokens_that_share_a_warp(tokens):
    check(tokens, "bf16", 2, 1, 128, tokens, (128, 1, False), per_head=True)
    check(tokens, "bf16", 3, 1, 64, tokens, (64, 1, True))


@pytest.mark.parametrize("which", ["q", "k", "qk"])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_weights(which, per_head, offset):
    check(4, "bf16", 8, 2, 128, 19, (128, 1, False), per_head, which, offset=offset)


@pytest.mark.parametrize("size,eps", [(0.0, 1e-6), (2.0 ** -60, 2.0 ** -126), (2.0 ** 50, 1e-6), (1e-4, 1e-5)])
def test_sizes(size, eps):
    check(5, "bf16", 8, 2, 128, 19, (128, 1, False), size=size, eps=eps)
    check(6, "fp32", 4, 4, 64, 19, None, size=size, eps=eps)


def test_strides():
    check(7, "bf16", 8, 2, 128, 33, (128, 1, False), pad=24)
    check(8, "fp8", 8, 2, 128, 33, (64, 1, True), heads_first=True)
    check(9, "fp32", 8, 2, 128, 33, (64, 1, True), pad=4)


def test_in_place_and_captured():
    """q in place; a captured write reads weights, q and positions anew."""
    gen = R.generator(10)
    rotary, table = R.rotary_of((128, 1, False))
    q, k, v = (R.rows(gen, 12, h, 128, torch.bfloat16) for h in (8, 2, 2))
    pools = R.pool(gen, 2, 2, 128, "bf16")
    w = [N.weight(gen, (128,), torch.bfloat16) for _ in range(2)]
    norm = HeadNorm(*w)
    slots = torch.arange(12, dtype=torch.int32, device="cuda")
    positions = torch.arange(12, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv_write(k, v, *pools, slots, q=q, q_out=q, rotary=rotary, positions=positions, norm=norm)
    positions += 1000
    w[0].mul_(2.0)
    ref, pair = N.rows(q, w[0], rotary, table, positions)
    graph.replay()
    torch.cuda.synchronize()
    off = N.loose(ref, pair)
    assert ((q.double() - ref).abs() <= off + R.HALF[torch.bfloat16] * (ref.abs() + off)).all()


def test_what_is_refused():
    gen = R.generator(11)
    q, k, v = (R.rows(gen, 4, h, 128, torch.bfloat16) for h in (8, 2, 2))
    pools = R.pool(gen, 1, 2, 128, "bf16")
    slots = torch.arange(4, dtype=torch.int32, device="cuda")
    w = N.weight(gen, (128,), torch.bfloat16)
    for bad in (dict(), dict(q_weight=w.half()), dict(q_weight=w, k_weight=w.float()), dict(k_weight=w[:120:2]),
                dict(q_weight=w.cpu()), dict(k_weight=w[1:]), dict(q_weight=w.view(1, 1, -1)),
                dict(q_weight=w, k_weight=w[:64])):
        with pytest.raises(ValueError):
            HeadNorm(**bad)
    two = N.weight(gen, (4, 128), torch.bfloat16)
    for norm in (HeadNorm(w.float(), w.float()), HeadNorm(w[:64], w[:64]), HeadNorm(k_weight=two), HeadNorm(two)):
        with pytest.raises(ValueError):
            kv_write(k, v, *pools, slots, q=q, norm=norm)
    with pytest.raises(ValueError):
        kv_write(k, v, *pools, slots, norm=HeadNorm(w))
