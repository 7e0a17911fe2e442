"""What is measured: the operators of a serving step over a cache held in 4 bits,
and what fills such a cache, through the calls a serving program makes.

  attend  a decode step or a tree-masked prefill over a paged cache in 4 bits: e2m1
          values, an e4m3 scale for each 16 of them, an fp32 scale per kv head
  store   tokens moved into that cache (keys as they are, already at their
          positions) and read back
  write   the tokens of a step or of a prompt on their way into any cache: the norm
          of each head of q and k, then their rotation, then rounding
  slots   the slots and positions of the tokens that a batch of sequences adds,
          with pages from a free list, on the GPU from lengths and page tables
  serve   the four together: one step of the branches of a tree

A program keeps the plan, the pools, the page tables, the weights, the rotary table
and its outputs between steps, so they are part of the prepared state.  Lengths
depend on the case alone, the page order and the values on the seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
BLOCK = 16                       # elements that share a scale in the 4-bit cache
E4M3_MAX = 448.0
E2M1_MAX = 6.0
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
ROW_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.bfloat16, "fp4": torch.bfloat16}
ROW_BYTES = {"bf16": 2, "fp32": 4, "fp8": 2, "fp4": 2}
KV_BITS = {"bf16": 16, "fp32": 32, "fp8": 8, "fp4": 4.5}
EPS = 1e-6


def _named(name, case):
    return dict(case, name=name) if name else case


def _attend(name, kind, q_heads, kv_heads, requests, prefix, joined, threads_lo, threads_hi, leaves,
            own_lo, own_hi, cap, permuted, shape):
    """kind decode: `leaves` branches of own_lo .. own_hi tokens under each request's prefix.
    kind prefill: `leaves` chunks of own_lo .. own_hi tokens behind the prefix and `joined` threads."""
    return _named(name, dict(op="attend", kind=kind, mode="fp4", q_heads=q_heads, kv_heads=kv_heads,
                             head_dim=128, requests=requests, prefix=prefix, joined=joined,
                             threads_lo=threads_lo, threads_hi=threads_hi, leaves=leaves, own_lo=own_lo,
                             own_hi=own_hi, cap=cap, permuted=permuted, shape=shape))


def _store(name, kv_heads, tokens, runs):
    """`tokens` rows of `runs` threads, each a run of consecutive slots of its pages."""
    return _named(name, dict(op="store", mode="fp4", kv_heads=kv_heads, head_dim=128, tokens=tokens, runs=runs))


def _write(name, mode, q_heads, kv_heads, head_dim, tokens, padding, rotary_dim, axes, interleaved,
           unit_offset, first):
    """`tokens` rows, the last `padding` of them without a slot; positions from `first` on."""
    return _named(name, dict(op="write", mode=mode, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                             tokens=tokens, padding=padding, rotary_dim=rotary_dim, axes=axes,
                             interleaved=interleaved, unit_offset=unit_offset, first=first))


def _slots(name, seqs, held_lo, held_hi, new_lo, new_hi, spare, given, shape):
    """`seqs` sequences that hold held_lo .. held_hi tokens and add new_lo .. new_hi; outputs have
    `spare` rows more than tokens.  given: new pages from a free list (else the tables have them)."""
    return _named(name, dict(op="slots", mode="bf16", seqs=seqs, held_lo=held_lo, held_hi=held_hi,
                             new_lo=new_lo, new_hi=new_hi, spare=spare, given=given, shape=shape))


def _serve(name, q_heads, kv_heads, prefix, leaves, own_lo, own_hi, shape):
    """A step of `leaves` branches of own_lo .. own_hi tokens, the step's one among them, under one prefix."""
    return _named(name, dict(op="serve", kind="decode", mode="fp4", q_heads=q_heads, kv_heads=kv_heads,
                             head_dim=128, requests=1, prefix=prefix, joined=0, threads_lo=0, threads_hi=0,
                             leaves=leaves, own_lo=own_lo, own_hi=own_hi, cap=0.0, permuted=True, shape=shape,
                             rotary_dim=128, axes=1, interleaved=False, unit_offset=False))


def listed():
    return [
        # the smallest step: one short request that has just forked; launches and latency count
        _attend("attend_tiny", "decode", 8, 2, 1, 256, 0, 0, 0, 4, 64, 64, 0.0, False, 0),
        # one request with 16 trials of ragged length, the common single-user step
        _attend("attend_trials16", "decode", 32, 8, 1, 2048, 0, 0, 0, 16, 512, 4096, 0.0, False, 1),
        # long reasoning, what a 4-bit cache is for: a long prefix, many long branches
        _attend("attend_long", "decode", 64, 8, 1, 16384, 0, 0, 0, 32, 4096, 8192, 0.0, True, 4),
        # thread openings: 16 chunks of 64 tokens prefilled under a shared prefix
        _attend("attend_fork", "prefill", 32, 8, 1, 2048, 0, 0, 0, 16, 64, 64, 0.0, False, 6),
        # the join: new text prefilled over the prefix and 16 finished threads
        _attend("attend_join", "prefill", 32, 8, 1, 2048, 16, 512, 4096, 1, 1024, 1024, 0.0, True, 1),
        # one finished thread moved into the 4-bit cache
        _store("store_thread", 8, 777, 1),
        # 16 finished threads of a join moved into it
        _store("store_join", 8, 38803, 16),
        # the tokens of one decode step of 16 branches, bf16 cache
        _write("write_step", "bf16", 32, 8, 128, 16, 0, 128, 1, False, False, 6000),
        # a batch of prompts padded to a fixed size, cache in e4m3
        _write("write_batch_e4m3", "fp8", 32, 8, 128, 8192, 200, 128, 1, False, False, 0),
        # a decode step of 64 branches, every one a token further
        _slots("slots_step", 64, 512, 8192, 1, 1, 0, True, 2),
        # prompts of 256 requests, ragged, padded to a fixed size
        _slots("slots_prompts", 256, 0, 64, 64, 800, 777, True, 3),
        # one step of 16 branches as a program runs it: slots, norms and rotation, write, attention
        _serve("serve_trials16", 32, 8, 2048, 16, 512, 4096, 1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.random()
    heads = rng.choice([(8, 2), (32, 8), (64, 8), (28, 4), (16, 16), (5, 1), (40, 8)])
    if op < 0.14:
        kv_heads = rng.randint(1, 16)
        tokens = _log(rng, 1, min(38803, 38803 * 8 // kv_heads))
        return _store(None, kv_heads, tokens, _log(rng, 1, min(tokens, 64)))
    if op < 0.34:
        mode = rng.choice(["bf16", "bf16", "fp8", "fp8", "fp32"])
        head_dim = 128 if mode == "fp8" else rng.choice([64, 128])
        tokens = _log(rng, 1, 8192 * 48 * 128 // ((heads[0] + 2 * heads[1]) * head_dim * (2 if mode == "fp32" else 1)))
        return _write(None, mode, *heads, head_dim, tokens, rng.choice([0, rng.randrange(tokens)]),
                      16 * rng.randint(1, head_dim // 16), rng.choice([1, 1, 2, 3]), rng.random() < 0.4,
                      rng.random() < 0.3, _log(rng, 1, 1000000))
    if op < 0.48:
        seqs = _log(rng, 1, 2048)
        most = 110000 // seqs
        hi = rng.choice([1, _log(rng, 1, most)])
        held = _log(rng, 1, 16384)
        return _slots(None, seqs, rng.choice([0, held // 2]), held, rng.choice([0 if seqs > 8 else 1, 1, hi]), hi,
                      rng.choice([0, _log(rng, 1, 1000)]), rng.random() < 0.7, rng.randrange(1 << 30))
    shape = rng.randrange(1 << 30)
    cap = rng.choice([0.0, 0.0, 0.0, 50.0])
    if op < 0.7:
        joined = rng.choice([0, 0, _log(rng, 1, 16)])
        tlo = _log(rng, 16, 1024) if joined else 0
        chunks = rng.choice([1, 1, 2, _log(rng, 2, 32)])
        lo = _log(rng, 1, 1024 // chunks)
        case = _attend(None, "prefill", *heads, 1, _log(rng, 1, 8192), joined, tlo,
                       _log(rng, tlo, 2048) if joined else 0, chunks, lo, _log(rng, lo, 1024 // chunks), cap,
                       rng.random() < 0.5, shape)
    elif op < 0.93:
        lo = _log(rng, 1, 4096)
        case = _attend(None, "decode", *heads, _log(rng, 1, 8), _log(rng, 16, 16384), 0, 0, 0, _log(rng, 1, 48),
                       lo, _log(rng, lo, 8192), cap, rng.random() < 0.5, shape)
    else:
        lo = _log(rng, 1, 4096)
        case = _serve(None, *heads, _log(rng, 16, 8192), _log(rng, 1, 48), lo, _log(rng, lo, 8192), shape)
    # no larger than the listed cases (the plain form holds every path's keys apart)
    while True:
        paths = case["requests"] * case["leaves"] * case["kv_heads"] * (
            case["prefix"] + case["joined"] * case["threads_hi"] + case["own_hi"])
        if (work(case)["flops"] <= 6e11 and paths <= 32 * 8 * 24576
                and (case["kind"] == "decode" or paths * case["own_hi"] <= 8 * 1024 * 42000)):
            return case
        key = max(("requests", "leaves", "own_hi", "prefix", "joined"),
                  key=lambda k: case[k] / {"requests": 4, "leaves": 8, "joined": 4}.get(k, 512))
        case[key] = max(1, int(case[key] * 0.7))
        case["own_lo"] = min(case["own_lo"], case["own_hi"])


# ------------------------------------------------------------------ the 4-bit cache

def _codes(y):
    """e2m1 codes 0 .. 15 of y (to nearest, ties to the even code, 6 at most), NaN aside."""
    a = y.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return c | (torch.signbit(y).to(torch.uint8) << 3)


def _packed(x, scale):
    """x [..., d] in 32 bits with its head's scale [..., 1] as (values [..., d / 2], block scales
    [..., d / 16]), bytes: s = e4m3(max |x| / (6 scale)), codes e2m1(x / (s scale)), each quotient a
    product with the rounded reciprocal."""
    b = x.unflatten(-1, (-1, BLOCK))
    s = (b.abs().amax(dim=-1) * (1.0 / (E2M1_MAX * scale))).clamp(max=E4M3_MAX).to(torch.float8_e4m3fn)
    step = s.float() * scale
    y = torch.where(step > 0, 1.0 / step, torch.zeros_like(step))
    c = _codes(b * y.unsqueeze(-1)).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), s.view(torch.uint8)


def _page_bytes(d):
    """Bytes of a page of one kv head: 16 rows of d / 2 bytes of values, then 16 of d / 16 scales."""
    return PAGE * (d // 2 + d // BLOCK)


def _pool4(gen, pages, case):
    """K and V pools in 4 bits of N(0, 1) values with some larger channels, and their head scales."""
    h, d = case["kv_heads"], case["head_dim"]
    pools, scales = [], []
    for _ in range(2):
        gain = torch.exp(0.4 * torch.randn((h, 1, d), generator=gen, device="cuda"))
        scale = 4.5 * gain.amax(dim=(1, 2)) / (E4M3_MAX * E2M1_MAX)
        pool = torch.empty((pages, h, _page_bytes(d)), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 24) // (h * PAGE * d))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = torch.randn((n, h, PAGE, d), generator=gen, device="cuda") * gain
            v, s = _packed(x, scale.view(-1, 1, 1))
            pool[p:p + n, :, :PAGE * d // 2] = v.flatten(2)
            pool[p:p + n, :, PAGE * d // 2:] = s.flatten(2)
        pools.append(pool)
        scales.append(scale)
    return pools[0], pools[1], scales[0], scales[1]


def _rows4(pages, scale, slots, dtype):
    """Rows [..., H_kv, d] of the slots [...] of a 4-bit pool, in `dtype`."""
    d = pages.shape[2] // 9
    page, at = slots // PAGE, slots % PAGE
    v = pages[..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))[page, :, at]
    s = pages[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // BLOCK))[page, :, at].view(torch.float8_e4m3fn)
    table = torch.tensor(E2M1 + [-x for x in E2M1], dtype=dtype, device="cuda")
    x = table[torch.stack([v & 15, v >> 4], dim=-1).flatten(-2).long()]
    s = s.to(torch.float32).to(dtype) * scale.to(dtype).view(-1, 1)
    return (x.unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2)


def _put4(pages, page, at, x, scale):
    """Rows x [n, H_kv, d] in 32 bits into slots (page, at) of a 4-bit pool."""
    d = x.shape[-1]
    v, s = _packed(x, scale.view(-1, 1))
    pages[..., :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))[page, :, at] = v
    pages[..., PAGE * d // 2:].unflatten(-1, (PAGE, d // BLOCK))[page, :, at] = s


# ------------------------------------------------------------------ inputs

def _forest(case):
    """(parent, node lengths, leaf or chunk nodes) of an attend or serve case."""
    rng = np.random.default_rng(case["shape"])
    parent, lens, leaves = [], [], []

    def node(up, lo, hi):
        parent.append(up)
        lens.append(int(rng.integers(lo, hi + 1)))
        return len(parent) - 1

    for _ in range(case["requests"]):
        up = node(-1, case["prefix"], case["prefix"])
        for _ in range(case["joined"]):
            up = node(up, case["threads_lo"], case["threads_hi"])
        leaves += [node(up, case["own_lo"], case["own_hi"]) for _ in range(case["leaves"])]
    return parent, lens, leaves


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _tree(case, seed):
    parent, lens, leaves = _forest(case)
    pages = [-(-n // PAGE) for n in lens]
    ptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    ids = np.arange(ptr[-1], dtype=np.int32)
    if case["permuted"]:
        ids = np.random.default_rng(seed).permutation(ids).astype(np.int32)
    return dict(parent=parent, lens=lens, leaves=leaves, ptr=ptr, ids=ids)


def _tree_inputs(case, seed):
    """An attend case's tree, page table, q and pools."""
    t = _tree(case, seed)
    gen = _generator(seed)
    queries = sum(t["lens"][n] for n in t["leaves"]) if case["kind"] == "prefill" else len(t["leaves"])
    q = torch.randn((queries, case["q_heads"], case["head_dim"]), generator=gen, device="cuda").to(torch.bfloat16)
    k_pages, v_pages, k_scale, v_scale = _pool4(gen, max(1, int(t["ptr"][-1])), case)
    return dict(t, q=q, k_pages=k_pages, v_pages=v_pages, k_scale=k_scale, v_scale=v_scale)


def _path(t, n):
    path = []
    while n >= 0:
        path.append(n)
        n = t["parent"][n]
    return path[::-1]


def _node_slots(t, n):
    pages = t["ids"][t["ptr"][n]:t["ptr"][n + 1]].astype(np.int64)
    return (pages[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:t["lens"][n]]


def _index(case, t):
    """The index arrays of a padded batch: a row per leaf (or chunk) with the
    slots of its path, the q row of each of its queries and how many keys it sees."""
    prefill = case["kind"] == "prefill"
    paths = [np.concatenate([_node_slots(t, m) for m in _path(t, n)]) for n in t["leaves"]]
    rows = [t["lens"][n] if prefill else 1 for n in t["leaves"]]
    keys, most = max(len(p) for p in paths), max(rows)
    slots = np.zeros((len(paths), keys), dtype=np.int64)
    q_row = np.zeros((len(paths), most), dtype=np.int64)
    seen = np.ones((len(paths), most), dtype=np.int64)
    pick = np.zeros(sum(rows), dtype=np.int64)
    at = 0
    for i, (p, r) in enumerate(zip(paths, rows)):
        slots[i, :len(p)] = p
        q_row[i, :r] = np.arange(at, at + r)
        seen[i, :r] = len(p) - r + 1 + np.arange(r) if prefill else len(p)
        pick[at:at + r] = i * most + np.arange(r)
        at += r
    return {k: torch.from_numpy(x).cuda() for k, x in
            dict(path_slots=slots, q_row=q_row, seen=seen, pick=pick).items()}


def _freqs(case):
    half = case["rotary_dim"] // 2
    return (1e6 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()


def _axes(case):
    """Axis of each frequency: equal contiguous sections."""
    half = case["rotary_dim"] // 2
    return [min(i * case["axes"] // half, case["axes"] - 1) for i in range(half)]


def _rows(gen, case, n):
    """q, k and v rows (views of one projection's output, as a model has them)."""
    h_q, h_kv, d = case.get("q_heads", 0), case["kv_heads"], case["head_dim"]
    qkv = torch.randn((n, (h_q + 2 * h_kv) * d), generator=gen, device="cuda")
    # keys of real models have a few large channels; every head has a magnitude of its own
    qkv *= torch.exp(0.5 * torch.randn(h_q + 2 * h_kv, generator=gen, device="cuda")).repeat_interleave(d)
    qkv = qkv.to(ROW_DTYPE[case["mode"]])
    return (x.view(n, -1, d) for x in qkv.split([h_q * d, h_kv * d, h_kv * d], dim=1))


def _weights(gen, case):
    """The norms' weights of q and of k (for unit_offset: what is added to 1)."""
    base = 0.0 if case["unit_offset"] else 1.0
    return tuple((base + 0.2 * torch.randn(case["head_dim"], generator=gen, device="cuda")).to(ROW_DTYPE[case["mode"]])
                 for _ in range(2))


def _table_slots(rng, pages, n):
    """Slots of n tokens in pages of a random order."""
    mine = rng.permutation(pages)[:-(-n // PAGE)]
    return (mine[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:n]


def _store_inputs(case, seed):
    gen = _generator(seed)
    _, k, v = _rows(gen, dict(case, q_heads=0), case["tokens"])
    n, runs = case["tokens"], case["runs"]
    sizes = [n * (i + 1) // runs - n * i // runs for i in range(runs)]
    pages = sum(-(-s // PAGE) for s in sizes)
    order, slots = np.random.default_rng(seed).permutation(pages), []
    for s in sizes:
        mine, order = order[:-(-s // PAGE)], order[-(-s // PAGE):]
        slots.append((mine[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:s])
    # scales from other text: a little small or large for the largest values
    scales = [x.float().abs().amax(dim=(0, 2)) / (E4M3_MAX * E2M1_MAX)
              * (0.9 + 0.2 * torch.rand(case["kv_heads"], generator=gen, device="cuda")) for x in (k, v)]
    pools = [torch.zeros((pages, case["kv_heads"], _page_bytes(case["head_dim"])), dtype=torch.uint8, device="cuda")
             for _ in range(2)]
    return dict(k=k, v=v, k_pages=pools[0], v_pages=pools[1], k_scale=scales[0], v_scale=scales[1],
                slots=torch.from_numpy(np.concatenate(slots).astype(np.int32)).cuda())


def _write_inputs(case, seed):
    gen, mode = _generator(seed), case["mode"]
    n, live, d = case["tokens"], case["tokens"] - case["padding"], case["head_dim"]
    q, k, v = _rows(gen, case, n)
    weights = _weights(gen, case)
    pages = -(-live // PAGE) + 1 + live // (8 * PAGE)
    k_scale = v_scale = None
    pools = [torch.randn((pages, case["kv_heads"], PAGE, d), generator=gen, device="cuda") for _ in range(2)]
    pools = [x.clamp(-4, 4).to(torch.float8_e4m3fn) if mode == "fp8" else x.to(ROW_DTYPE[mode]) for x in pools]
    if mode == "fp8":           # a normed head's elements reach about 5 times the weight; v as scales from other text
        k_scale = torch.full((case["kv_heads"],), 6.0 / E4M3_MAX, device="cuda")
        v_scale = v.float().abs().amax(dim=(0, 2)) * 0.9 / E4M3_MAX
    rng = np.random.default_rng(seed)
    slots = np.full(n, -1, dtype=np.int32)
    slots[:live] = _table_slots(rng, pages, live)
    # one axis: running positions; several: time runs, the others walk over an image grid
    step = case["first"] + np.arange(n, dtype=np.int64)
    positions = np.stack([step, case["first"] + step // 32 % 32, case["first"] + step % 32][:case["axes"]])
    return dict(q=q, k=k, v=v, weights=weights, k_pages=pools[0], v_pages=pools[1], k_scale=k_scale,
                v_scale=v_scale, slots=torch.from_numpy(slots).cuda(),
                positions=torch.from_numpy(positions.astype(np.int32)).cuda(), live=live)


def _lengths(case):
    """(held, new) tokens of a slots case's sequences."""
    rng = np.random.default_rng(case["shape"])
    return (rng.integers(case["held_lo"], case["held_hi"] + 1, case["seqs"]),
            rng.integers(case["new_lo"], case["new_hi"] + 1, case["seqs"]))


def _slots_inputs(case, seed):
    held, new = _lengths(case)
    rng = np.random.default_rng(seed)
    had, have = -(-held // PAGE), -(-(held + new) // PAGE)
    pages = rng.permutation(int(have.sum()) + 64).astype(np.int32)
    table = np.full((case["seqs"], int(have.max()) + 1), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(had if case["given"] else have):
        table[r, :n] = pages[at:at + n]
        at += n
    first = rng.integers(0, 4096, case["seqs"])          # tokens of the nodes above
    arrays = dict(page_table=table, held=held, new=new, first=first, free_pages=pages[at:],
                  free_used=np.array([5 if case["given"] else 0]))
    return {k: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda() for k, x in arrays.items()}


def _serve_inputs(case, seed):
    """A tree whose branches' last tokens are the step's: their rows, and the page tables before it."""
    s = _tree_inputs(case, seed)
    gen, leaves = _generator(seed + 1), s["leaves"]
    s["q"], s["k"], s["v"] = _rows(gen, case, len(leaves))
    s["weights"] = _weights(gen, case)
    own_len = np.array([s["lens"][n] for n in leaves])
    table = np.full((len(leaves), int((-(-own_len // PAGE)).max())), -1, dtype=np.int32)
    opened = []
    for r, n in enumerate(leaves):
        pages = s["ids"][s["ptr"][n]:s["ptr"][n + 1]]
        table[r, :len(pages)] = pages
        if s["lens"][n] % PAGE == 1:                     # the step's token opens its last page
            table[r, len(pages) - 1] = -1
            opened.append(pages[-1])
    arrays = dict(page_table=table, held=own_len - 1, first=np.full(len(leaves), case["prefix"]),
                  free_pages=np.array(opened + [0]), free_used=np.zeros(1))
    s.update({k: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda() for k, x in arrays.items()})
    return s


def _plan(case, t):
    from paper_2608_24658_gb300.api import Plan
    return Plan(num_q_heads=case["q_heads"], num_kv_heads=case["kv_heads"], head_dim=case["head_dim"],
                mode="fp4", parent=t["parent"], node_len=t["lens"], node_page_ptr=t["ptr"],
                page_ids=t["ids"], leaf_node=t["leaves"], num_physical_pages=t["k_pages"].shape[0],
                prefill=case["kind"] == "prefill", logit_cap=case["cap"])


def prepare(case, seed):
    op = case["op"]
    state = {"case": case}
    if op == "slots":
        state.update(_slots_inputs(case, seed))
        held, new = _lengths(case)
        n = int(new.sum()) + case["spare"]
        state.update({k: torch.empty(n, dtype=torch.int32, device="cuda") for k in ("slots", "positions")})
        state["token_ptr"] = torch.empty(case["seqs"] + 1, dtype=torch.int32, device="cuda")
        state["lens_out"], state["used_out"] = torch.empty_like(state["held"]), torch.empty_like(state["free_used"])
        return state
    if op == "store":
        state.update(_store_inputs(case, seed))
        state["k_out"], state["v_out"] = (torch.empty((case["tokens"], case["kv_heads"], case["head_dim"]),
                                                      dtype=torch.bfloat16, device="cuda") for _ in range(2))
        return state
    if op in ("attend", "serve"):
        state.update((_tree_inputs if op == "attend" else _serve_inputs)(case, seed))
        q = state["q"]
        state.update(out=torch.empty(q.shape, dtype=q.dtype, device="cuda"),
                     lse=torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"))
        # what either form keeps between steps: the library its plan, the plain form its index arrays
        if own:
            state["plan"] = _plan(case, state)
            state["workspace"] = state["plan"].workspace(q.device)
        else:
            state.update(_index(case, state))
        if op == "attend":
            return state
        n = len(state["leaves"])
        state.update({k: torch.empty(n, dtype=torch.int32, device="cuda") for k in ("slots", "positions")})
        state["live"] = n
    else:
        state.update(_write_inputs(case, seed))
    state["q_out"] = torch.empty_like(state["q"], memory_format=torch.contiguous_format)
    state["inv_freq"] = _freqs(case)
    state["axes"] = torch.tensor(_axes(case), device="cuda")
    if own:
        from paper_2608_24658_gb300.api import HeadNorm, Rotary
        state["rotary"] = Rotary(state["inv_freq"], axes=_axes(case), interleaved=case["interleaved"])
        state["norm"] = HeadNorm(*state["weights"], eps=EPS, unit_offset=case["unit_offset"])
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"attend": _attend_own, "store": _store_own, "write": _write_own, "slots": _slots_own,
                "serve": _serve_own}[op](state)
    return {"attend": _attend_plain, "store": _store_plain, "write": _write_plain, "slots": _slots_plain,
            "serve": _serve_plain}[op](state)


def _attend_own(s):
    return s["plan"].decode(s["q"], s["k_pages"], s["v_pages"], out=s["out"], lse=s["lse"],
                            workspace=s["workspace"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _store_own(s):
    from paper_2608_24658_gb300.api import kv_read, kv_write
    kv_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slots"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return kv_read(s["k_pages"], s["v_pages"], s["slots"], k=s["k_out"], v=s["v_out"], k_scale=s["k_scale"],
                   v_scale=s["v_scale"])


def _write_own(s):
    from paper_2608_24658_gb300.api import kv_write
    q_out = kv_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slots"], q=s["q"], q_out=s["q_out"],
                     norm=s["norm"], rotary=s["rotary"], positions=s["positions"], k_scale=s["k_scale"],
                     v_scale=s["v_scale"])
    return {"q": q_out, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _slots_own(s):
    from paper_2608_24658_gb300.api import kv_slots
    given = s["case"]["given"]
    kv_slots(s["page_table"], s["held"], s["new"], first=s["first"],
             free_pages=s["free_pages"] if given else None, free_used=s["free_used"] if given else None,
             used_out=s["used_out"] if given else None, slots=s["slots"], positions=s["positions"],
             token_ptr=s["token_ptr"], lens_out=s["lens_out"])
    return {k: s[k] for k in ("slots", "positions", "token_ptr", "lens_out", "page_table")} | (
        {"used": s["used_out"]} if given else {})


def _serve_own(s):
    from paper_2608_24658_gb300.api import kv_slots, kv_write
    kv_slots(s["page_table"], s["held"], first=s["first"], free_pages=s["free_pages"],
             free_used=s["free_used"], slots=s["slots"], positions=s["positions"])
    q = kv_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slots"], q=s["q"], q_out=s["q_out"],
                 norm=s["norm"], rotary=s["rotary"], positions=s["positions"], k_scale=s["k_scale"],
                 v_scale=s["v_scale"])
    out, lse = s["plan"].decode(q, s["k_pages"], s["v_pages"], out=s["out"], lse=s["lse"],
                                workspace=s["workspace"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return {"slots": s["slots"], "positions": s["positions"], "out": out, "lse": lse}


def _attend_plain(s):
    case = s["case"]
    h_q, h_kv, d, cap = case["q_heads"], case["kv_heads"], case["head_dim"], case["cap"]
    g = h_q // h_kv
    n, most = s["q_row"].shape
    k = _rows4(s["k_pages"], s["k_scale"], s["path_slots"], torch.float32)            # [n, keys, H_kv, d]
    q = s["q"][s["q_row"]].float().view(n, most, h_kv, g, d).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(n, h_kv, g * most, d), k.permute(0, 2, 3, 1)) / math.sqrt(d)
    x = cap * torch.tanh(x / cap) if cap else x
    hidden = torch.arange(k.shape[1], device="cuda") >= s["seen"].unsqueeze(-1)       # [n, most, keys]
    x = x.view(n, h_kv, g, most, -1).masked_fill(hidden[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(dim=-1, keepdim=True)
    v = _rows4(s["v_pages"], s["v_scale"], s["path_slots"], torch.float32)
    o = torch.matmul(p.view(n, h_kv, g * most, -1), v.permute(0, 2, 1, 3)).view(n, h_kv, g, most, d) / l
    o = o.permute(0, 3, 1, 2, 4).reshape(n * most, h_q, d)[s["pick"]]
    lse = (m + torch.log(l)).permute(0, 3, 1, 2, 4).reshape(n * most, h_q)[s["pick"]]
    return o.to(s["q"].dtype), lse


def _store_plain(s):
    slots = s["slots"].long()
    result = []
    for pages, rows, scale in ((s["k_pages"], s["k"], s["k_scale"]), (s["v_pages"], s["v"], s["v_scale"])):
        _put4(pages, slots // PAGE, slots % PAGE, rows.float(), scale)
        result.append(_rows4(pages, scale, slots, torch.float32).to(torch.bfloat16))
    return tuple(result)


def _normed(x, w, case):
    x, w = x.float(), w.float() + (1.0 if case["unit_offset"] else 0.0)
    return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w


def _turned(x, cos, sin, case):
    """x [tokens, heads, d] in 32 bits with its first rotary_dim dims rotated."""
    r = case["rotary_dim"]
    head, rest = x.split([r, x.shape[2] - r], dim=2)
    if case["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), rest], dim=2)
    a, b = head.split(r // 2, dim=2)
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], dim=2)


def _write_plain(s):
    case, live = s["case"], s["live"]
    positions = s["positions"].view(case["axes"], -1)
    angle = positions[s["axes"]].t().double() * s["inv_freq"].double()      # [tokens, rotary_dim / 2]
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    slots = s["slots"][:live].long()
    page, at = slots // PAGE, slots % PAGE
    q, k = (_turned(_normed(s[x], w, case), cos, sin, case) for x, w in zip("qk", s["weights"]))
    for pages, rows, scale in ((s["k_pages"], k[:live], s["k_scale"]),
                               (s["v_pages"], s["v"][:live].float(), s["v_scale"])):
        if case["mode"] == "fp4":
            _put4(pages, page, at, rows, scale)
        elif case["mode"] == "fp8":
            rows = (rows / scale.view(-1, 1)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
            pages.view(torch.uint8)[page, :, at] = rows.view(torch.uint8)
        else:
            pages[page, :, at] = rows.to(pages.dtype)
    return {"q": q.to(s["q"].dtype), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _slots_of(s, new, tokens, given):
    """(slots, positions, token_ptr, lens, used); new pages go into the table."""
    held, table = s["held"].long(), s["page_table"]
    ptr = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0))
    lens, used = held + new, None
    if given:
        had = (held + PAGE - 1) // PAGE
        need = (lens + PAGE - 1) // PAGE - had
        upto = torch.cumsum(need, 0)
        used = s["free_used"] + upto[-1]
        col = torch.arange(table.shape[1], device="cuda")
        at = s["free_used"].long() + (upto - need).unsqueeze(1) + col - had.unsqueeze(1)
        fresh = (col >= had.unsqueeze(1)) & (col < (had + need).unsqueeze(1))
        table.copy_(torch.where(fresh, s["free_pages"][at.clamp(0, s["free_pages"].numel() - 1)], table))
    t = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(ptr[1:], t, right=True).clamp(max=new.numel() - 1)
    index = held[seq] + t - ptr[seq]
    live = t < ptr[-1]
    page = table[seq, (index // PAGE).clamp(max=table.shape[1] - 1)].long()
    slots = torch.where(live, page * PAGE + index % PAGE, -1).int()
    positions = torch.where(live, s["first"][seq] + index, 0).int()
    return slots, positions, ptr.int(), lens.int(), used


def _slots_plain(s):
    given = s["case"]["given"]
    slots, positions, ptr, lens, used = _slots_of(s, s["new"].long(), s["slots"].numel(), given)
    return {"slots": slots, "positions": positions, "token_ptr": ptr, "lens_out": lens,
            "page_table": s["page_table"]} | ({"used": used.int()} if given else {})


def _serve_plain(s):
    n = s["live"]
    slots, positions, _, _, _ = _slots_of(s, torch.ones(n, dtype=torch.int64, device="cuda"), n, True)
    step = dict(s, slots=slots, positions=positions)
    step["q"] = _write_plain(step)["q"]
    out, lse = _attend_plain(step)
    return {"slots": slots, "positions": positions, "out": out, "lse": lse}


# ------------------------------------------------------------------ work

def _attend_work(case):
    h_kv, h_q, d = case["kv_heads"], case["q_heads"], case["head_dim"]
    parent, lens, leaves = _forest(case)
    under = [0] * len(parent)
    for i in leaves:
        under[i] = lens[i] if case["kind"] == "prefill" else 1
    queries = sum(under)
    for i in range(len(parent) - 1, 0, -1):
        if parent[i] >= 0:
            under[parent[i]] += under[i]
    mine = set(leaves) if case["kind"] == "prefill" else set()    # causal in the chunk itself
    keys = sum(lens[i] * (lens[i] + 1) // 2 if i in mine else lens[i] * under[i] for i in range(len(parent)))
    return {"bytes": int(sum(lens) * 2 * h_kv * d * KV_BITS["fp4"] / 8) + queries * h_q * (4 * d + 4) + 8 * h_kv,
            "flops": keys * h_q * 4 * d}


def work(case):
    op, mode = case["op"], case["mode"]
    if op == "attend":
        return _attend_work(case)
    if op == "slots":
        held, new = _lengths(case)
        tokens = int(new.sum())
        pages = -(-(held + new) // PAGE) - held // PAGE           # pages that the new tokens lie in
        return {"bytes": 4 * (4 * case["seqs"] + 1 + int(pages.sum()) + 2 * (tokens + case["spare"])),
                "flops": 4 * tokens}
    h_kv, d = case["kv_heads"], case["head_dim"]
    rb, kvb = ROW_BYTES[mode], KV_BITS[mode] / 8
    if op == "store":
        n = case["tokens"]
        return {"bytes": int(2 * n * h_kv * d * (2 * rb + kvb)) + 4 * n, "flops": 6 * n * h_kv * d}
    n = case["leaves"] if op == "serve" else case["tokens"]
    live, heads = n - case.get("padding", 0), h_kv + case["q_heads"]
    w = {"bytes": int((case["q_heads"] * n * 2 * rb + live * 2 * h_kv * (rb + kvb)) * d) + n * 4 * (1 + case["axes"]),
         "flops": n * heads * (4 * d + 3 * case["rotary_dim"])}
    if op == "serve":
        a = _attend_work(case)
        return {k: w[k] + a[k] for k in w}
    return w


# ------------------------------------------------------------------ in 64 bits

def _wide(x):
    return x.to(torch.float32).to(torch.float64)


def _exact_attention(case, t, q):
    """Attention of rows q [queries, H_q, d] (64 bits) over the tree t, path by path."""
    h_q, h_kv, d, cap = case["q_heads"], case["kv_heads"], case["head_dim"], case["cap"]
    g = h_q // h_kv
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device="cuda")
    row = 0
    for leaf in t["leaves"]:
        slots = torch.from_numpy(np.concatenate([_node_slots(t, n) for n in _path(t, leaf)])).cuda()
        k, v = (_rows4(t[x + "_pages"], t[x + "_scale"], slots, torch.float64).transpose(0, 1) for x in "kv")
        queries = t["lens"][leaf] if case["kind"] == "prefill" else 1
        total = k.shape[1]
        for t0 in range(0, queries, 128):
            t1 = min(queries, t0 + 128)
            for h in range(h_kv):
                x = torch.einsum("tgd,kd->gtk", q[row + t0:row + t1, h * g:(h + 1) * g], k[h]) / math.sqrt(d)
                x = cap * torch.tanh(x / cap) if cap else x
                if queries > 1:
                    last = total - queries + torch.arange(t0, t1, device="cuda")
                    x.masked_fill_(torch.arange(total, device="cuda") > last[:, None], -math.inf)
                z = torch.logsumexp(x, dim=-1)
                lse[row + t0:row + t1, h * g:(h + 1) * g] = z.t()
                out[row + t0:row + t1, h * g:(h + 1) * g] = torch.einsum(
                    "gtk,kd->tgd", torch.exp(x - z.unsqueeze(-1)), v[h])
        row += queries
    return out, lse


def _exact_attend(case, seed):
    t = _tree_inputs(case, seed)
    return _exact_attention(case, t, _wide(t["q"]))


def _nearest(x, bits, least, most):
    """x >= 0 to `bits` significant bits, but no finer than `least`, to nearest and even; at most `most`."""
    unit = torch.exp2(torch.floor(torch.log2(x.clamp(min=1e-300))) - (bits - 1)).clamp(min=least)
    return (torch.round(x / unit) * unit).clamp(max=most)


def _exact_store(case, seed):
    s = _store_inputs(case, seed)
    result = []
    for x, scale in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])):
        x = _wide(x).unflatten(-1, (-1, BLOCK)) / _wide(scale).view(-1, 1, 1)
        step = _nearest(x.abs().amax(dim=-1, keepdim=True) / E2M1_MAX, 4, 2.0 ** -9, E4M3_MAX)
        x = torch.where(step > 0, x / step, torch.zeros_like(x))
        x = torch.sign(x) * _nearest(x.abs(), 2, 0.5, E2M1_MAX) * step * _wide(scale).view(-1, 1, 1)
        result.append(x.flatten(-2))
    return tuple(result)


def _exact_rows(case, s, positions):
    """q and k normed and rotated, in 64 bits."""
    r, freqs, axes = case["rotary_dim"], _freqs(case).double(), _axes(case)
    n = s["k"].shape[0]
    turn = torch.polar(torch.ones(n, len(axes), dtype=torch.float64, device="cuda"),
                       torch.stack([positions[a].double() * f for a, f in zip(axes, freqs)], dim=1)).unsqueeze(1)
    result = []
    for x, w in zip((s["q"], s["k"]), s["weights"]):
        x = _wide(x)
        x = x / torch.sqrt(x.square().sum(dim=-1, keepdim=True) / x.shape[-1] + EPS)
        x = x * (_wide(w) + (1.0 if case["unit_offset"] else 0.0))
        first, second = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        first.copy_(z.real), second.copy_(z.imag)
        result.append(x)
    return result


def _exact_write(case, seed):
    s = _write_inputs(case, seed)
    q, k = _exact_rows(case, s, s["positions"])
    result = {"q": q}
    slots = s["slots"][s["slots"] >= 0].long()
    for name, rows in (("k", k), ("v", _wide(s["v"]))):
        pages, scale = _wide(s[name + "_pages"]), s[name + "_scale"]
        if scale is not None:
            rows = (rows / _wide(scale).view(-1, 1)).clamp(-E4M3_MAX, E4M3_MAX)
        pages[slots // PAGE, :, slots % PAGE] = rows[:len(slots)]
        result[name + "_pages"] = pages
    return result


def _exact_serve(case, seed):
    s = _serve_inputs(case, seed)
    last = [s["lens"][n] - 1 for n in s["leaves"]]
    slots = torch.tensor([_node_slots(s, n)[-1] for n in s["leaves"]], device="cuda")
    positions = torch.tensor([case["prefix"] + i for i in last], device="cuda")
    q, k = _exact_rows(case, s, positions.unsqueeze(0))
    for name, rows in (("k", k), ("v", _wide(s["v"]))):
        _put4(s[name + "_pages"], slots // PAGE, slots % PAGE, rows.float(), s[name + "_scale"])
    out, lse = _exact_attention(case, s, _wide(q.to(s["q"].dtype)))     # queries are rows of the model's type
    return {"slots": None, "positions": None, "out": out, "lse": lse}


def exact(case, seed):
    if case["op"] == "slots":                            # whole numbers
        return None
    return {"attend": _exact_attend, "store": _exact_store, "write": _exact_write,
            "serve": _exact_serve}[case["op"]](case, seed)
