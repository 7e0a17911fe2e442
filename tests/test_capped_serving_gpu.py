"""The cache operators and the capped attention together, as a serving program
runs a layer: scales from the prompt, the prompt written and prefilled, threads
forked and decoded token by token, and a finished thread moved behind the prompt."""
import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan, kv_read, kv_scales, kv_write
from tests import cap_ref as C
from tests import kv_ref as R

pytestmark = pytest.mark.gpu

H_Q, H_KV, D, CAP, PAGES = 8, 2, 128, 20.0, 64


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


class Cache:
    """Pools, a free list, and the page lists of nodes."""

    def __init__(self, mode, gen):
        self.mode, self.gen = mode, gen
        self.pools = R.pool(gen, PAGES, H_KV, D, mode)           # random bits, NaN among them
        self.free = list(np.random.default_rng(3).permutation(PAGES))
        self.parent, self.length, self.pages = [], [], []
        self.scales = dict(k_scale=None, v_scale=None)

    def node(self, parent, tokens):
        self.parent.append(parent)
        self.length.append(0)
        self.pages.append([])
        self.grow(len(self.parent) - 1, tokens)
        return len(self.parent) - 1

    def grow(self, n, tokens=1):
        self.length[n] += tokens
        opened = []
        while len(self.pages[n]) * R.PAGE < self.length[n]:
            opened.append(int(self.free.pop()))
            self.pages[n] += opened[-1:]
        return opened

    def slots(self, n, first=0):
        at = np.arange(first, self.length[n])
        return torch.tensor(np.array(self.pages[n])[at // R.PAGE] * R.PAGE + at % R.PAGE, dtype=torch.int32,
                            device="cuda")

    def tree(self, leaves, q):
        ptr = np.concatenate([[0], np.cumsum([len(p) for p in self.pages])]).astype(np.int32)
        return W.ForkTree(name="served", num_q_heads=H_Q, num_kv_heads=H_KV, head_dim=D, mode=self.mode,
                          parent=np.array(self.parent, np.int32), node_len=np.array(self.length, np.int32),
                          node_page_ptr=ptr, page_ids=np.array([p for ps in self.pages for p in ps], np.int32),
                          leaf_node=np.array(leaves, np.int32), num_physical_pages=PAGES, q=q,
                          k_pages=self.pools[0], v_pages=self.pools[1], **self.scales)


def projected(gen, tokens, dtype):
    """q, k, v of a fused projection."""
    x = torch.randn((tokens, (H_Q + 2 * H_KV) * D), generator=gen, device="cuda").to(dtype)
    return (y.unflatten(1, (-1, D)) for y in x.split([H_Q * D, H_KV * D, H_KV * D], dim=1))


@pytest.mark.parametrize("mode", ["bf16", "fp8"])
def test_a_layer_served(mode):
    gen = R.generator(31)
    cache = Cache(mode, gen)
    rotary, table = R.rotary_of((64, 3, False))
    prompt = 197
    q, k, v = projected(gen, prompt, torch.bfloat16)
    grid = torch.arange(prompt, dtype=torch.int32, device="cuda")
    pos = torch.stack([grid, grid // 16, grid % 16])
    if mode == "fp8":
        ks, vs = kv_scales(k, v, rotary=rotary)
        cache.scales = dict(k_scale=ks, v_scale=vs)
    root = cache.node(-1, prompt)
    q_out = kv_write(k, v, *cache.pools, cache.slots(root), q=q, rotary=rotary, positions=pos, **cache.scales)
    turned, size = R.rotated(q, rotary, table, pos)
    assert ((q_out.double() - turned).abs() <= R.bound(turned, size, torch.bfloat16)).all()
    tree = cache.tree([root], q_out)
    with Plan.for_prefill(tree, logit_cap=CAP) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    C.check(tree, CAP, out, lse, prefill=True)

    # three threads open; then every step appends a token to each of them
    leaves = [cache.node(root, n) for n in (1, 16, 30)]
    history = {n: [] for n in leaves}
    for n in leaves:
        _, k, v = projected(gen, cache.length[n], torch.bfloat16)
        at = prompt + torch.arange(cache.length[n], dtype=torch.int32, device="cuda")
        kv_write(k, v, *cache.pools, cache.slots(n), rotary=rotary, positions=at.expand(3, -1), **cache.scales)
        history[n].append((k, v))
    tree = cache.tree(leaves, torch.zeros((3, H_Q, D), dtype=torch.bfloat16, device="cuda"))
    with Plan.for_tree(tree, logit_cap=CAP) as plan:
        for step in range(20):
            q, k, v = projected(gen, 3, torch.bfloat16)
            at = torch.tensor([prompt + cache.length[n] for n in leaves], dtype=torch.int32, device="cuda")
            opened = [(cache.grow(n) or [-1])[0] for n in leaves]
            plan.append(opened)
            slots = torch.cat([cache.slots(n, cache.length[n] - 1) for n in leaves])
            q_out = kv_write(k, v, *cache.pools, slots, q=q, rotary=rotary, positions=at.expand(3, -1).contiguous(),
                             **cache.scales)
            for i, n in enumerate(leaves):
                history[n].append((k[i:i + 1], v[i:i + 1]))
            tree = cache.tree(leaves, q_out)
            out, lse = plan.decode_tree(tree)
            if step % 5 == 4:
                plan.check()
                C.check(tree, CAP, out, lse)

    # the join: the last thread's tokens move behind the first's, keys to their new positions
    first, last = leaves[0], leaves[2]
    shift = cache.length[first]
    k, v = kv_read(*cache.pools, cache.slots(last), **cache.scales)
    moved = cache.node(first, cache.length[last])
    by = torch.full((3, cache.length[last]), shift, dtype=torch.int32, device="cuda")
    kv_write(k, v, *cache.pools, cache.slots(moved), rotary=rotary, positions=by, **cache.scales)
    # against the thread's own keys, turned straight to where they are now
    raw = torch.cat([h[0] for h in history[last]])
    at = prompt + shift + torch.arange(cache.length[last], dtype=torch.int32, device="cuda")
    want, size = R.rotated(raw, rotary, table, at.expand(3, -1))
    got = C.node_kv(cache.tree([moved], q_out), moved)[0].transpose(0, 1)
    # two roundings to the cache's type (the second turns the first's errors within their
    # pairs: at most their sum), and one to bf16 between
    step = 2.0 ** -8 if mode == "bf16" else 2.0 ** -4 + 2.0 ** -8
    least = 0 if mode == "bf16" else 2.0 ** -9 * cache.scales["k_scale"].double().view(-1, 1)
    pair = torch.where(size > 0, size, raw.double().abs())
    assert ((got - want).abs() <= 1.01 * (2 * step * pair + 2 * least)).all()
    q, _, _ = projected(gen, 2, torch.bfloat16)
    tree = cache.tree([moved, leaves[1]], q.contiguous())
    with Plan.for_tree(tree, logit_cap=CAP) as plan:
        out, lse = plan.decode_tree(tree)
        plan.check()
    C.check(tree, CAP, out, lse)


@pytest.mark.parametrize("mode", ["bf16", "fp8", "fp32"])
def test_a_step_captured(mode):
    """Write and capped decode of a step in one graph, replayed with new rows and slots."""
    gen = R.generator(33)
    cache = Cache(mode, gen)
    dtype = R.ROWS[mode]
    rotary, table = R.rotary_of((128, 1, True))
    if mode == "fp8":
        cache.scales = {n: torch.full((H_KV,), 0.02, device="cuda") for n in ("k_scale", "v_scale")}
    root = cache.node(-1, 100)
    leaves = [cache.node(root, n) for n in (5, 17)]
    for n in range(3):
        _, k, v = projected(gen, cache.length[n], dtype)
        kv_write(k, v, *cache.pools, cache.slots(n), **cache.scales)
    q, k, v = (x.contiguous() for x in projected(gen, 2, dtype))
    slots = torch.cat([cache.slots(n, cache.length[n] - 1) for n in leaves])
    pos = torch.tensor([105, 117], dtype=torch.int32, device="cuda")
    q_out = torch.empty_like(q)
    out, lse = torch.empty_like(q), torch.empty((2, H_Q), device="cuda")
    tree = cache.tree(leaves, q_out)
    with Plan.for_tree(tree, logit_cap=CAP) as plan:
        workspace = plan.workspace(q.device)

        def step():
            kv_write(k, v, *cache.pools, slots, q=q, q_out=q_out, rotary=rotary, positions=pos, **cache.scales)
            plan.decode_tree(tree, out=out, lse=lse, workspace=workspace)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(4):
            for t, new in zip((q, k, v), projected(gen, 2, dtype)):
                t.copy_(new)
            pos += 1
            graph.replay()
            torch.cuda.synchronize()
            turned, size = R.rotated(q, rotary, table, pos)
            assert ((q_out.double() - turned).abs() <= R.bound(turned, size, dtype)).all()
            C.check(tree, CAP, out, lse)
        plan.check()
