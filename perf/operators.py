"""What is measured: the operators that surround and vary the attention of a
serving step, through the calls a serving program makes.

  attend  a decode step or a tree-masked prefill whose logits are capped by a
          tanh (s = c tanh(sm_scale <q, k> / c)), over a paged KV cache
  write   the tokens of a step or of a prompt: q and k rotated to their
          positions (one or several axes), k and v written into their slots of
          the paged cache, quantised when it holds e4m3
  read    the tokens of finished threads taken out of the cache again
  scales  the e4m3 scales per kv head of a batch of keys and values

A program keeps the plan, the pools, the rotary table and its outputs between
steps, so they are part of the prepared state.  Node lengths depend on the
case alone, the page order and the values on the seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
E4M3_MAX = 448.0
Q_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.bfloat16}
KV_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn}
Q_BYTES = {"bf16": 2, "fp32": 4, "fp8": 2}
KV_BYTES = {"bf16": 2, "fp32": 4, "fp8": 1}


def _attend(name, kind, mode, q_heads, kv_heads, head_dim, requests, prefix, joined, threads_lo,
            threads_hi, leaves, own_lo, own_hi, cap, gain, permuted, shape):
    """kind decode: `leaves` branches of own_lo .. own_hi tokens under each request's prefix.
    kind prefill: `leaves` chunks of own_lo .. own_hi tokens behind the prefix and `joined` threads.
    gain: standard deviation of the uncapped logits."""
    case = dict(op="attend", kind=kind, mode=mode, q_heads=q_heads, kv_heads=kv_heads,
                head_dim=head_dim, requests=requests, prefix=prefix, joined=joined,
                threads_lo=threads_lo, threads_hi=threads_hi, leaves=leaves, own_lo=own_lo,
                own_hi=own_hi, cap=cap, gain=gain, permuted=permuted, shape=shape)
    return dict(case, name=name) if name else case


def _write(name, mode, q_heads, kv_heads, head_dim, tokens, padding, with_q, rotary_dim, axes,
           interleaved, first):
    """`tokens` rows, the last `padding` of them without a slot; positions from `first` on."""
    case = dict(op="write", mode=mode, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                tokens=tokens, padding=padding, with_q=with_q, rotary_dim=rotary_dim, axes=axes,
                interleaved=interleaved, first=first)
    return dict(case, name=name) if name else case


def _read(name, mode, kv_heads, head_dim, tokens, runs):
    """`tokens` rows of `runs` threads, each a run of consecutive slots of its pages."""
    case = dict(op="read", mode=mode, kv_heads=kv_heads, head_dim=head_dim, tokens=tokens, runs=runs)
    return dict(case, name=name) if name else case


def _scales(name, kv_heads, tokens, rotary_dim, interleaved):
    case = dict(op="scales", mode="fp8", kv_heads=kv_heads, head_dim=128, tokens=tokens,
                rotary_dim=rotary_dim, interleaved=interleaved)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest step: one short request that has just forked; launches and latency count
        _attend("cap_tiny", "decode", "bf16", 8, 2, 64, 1, 256, 0, 0, 0, 4, 32, 64, 50.0, 1.0,
                False, 0),
        # one request with 16 trials of ragged length, the common single-user step
        _attend("cap_trials16", "decode", "bf16", 32, 8, 128, 1, 2048, 0, 0, 0, 16, 512, 4096,
                50.0, 1.0, False, 1),
        # long reasoning with the cache in e4m3, logits that reach the cap
        _attend("cap_long_e4m3", "decode", "fp8", 64, 8, 128, 1, 16384, 0, 0, 0, 32, 2048, 8192,
                30.0, 8.0, False, 4),
        # thread openings: 16 chunks of 64 tokens prefilled under a shared prefix
        _attend("cap_fork", "prefill", "bf16", 32, 8, 128, 1, 2048, 0, 0, 0, 16, 64, 64, 50.0,
                1.0, False, 6),
        # the join: new text prefilled over the prefix and 16 finished threads
        _attend("cap_join", "prefill", "bf16", 32, 8, 128, 1, 2048, 16, 512, 4096, 1, 1024, 1024,
                50.0, 1.0, False, 1),
        # the tokens of one decode step of 16 branches
        _write("write_step", "bf16", 32, 8, 128, 16, 0, True, 128, 1, False, 6000),
        # a prompt with images: three position axes (time, height, width), bf16 cache
        _write("write_prompt", "bf16", 32, 8, 128, 8192, 0, True, 128, 3, False, 0),
        # a batch padded to a fixed size, cache in e4m3, half of each head rotated in neighbouring pairs
        _write("write_batch_e4m3", "fp8", 64, 8, 128, 2500, 60, True, 64, 1, True, 100000),
        # one finished thread taken out of a bf16 cache
        _read("read_thread", "bf16", 8, 128, 777, 1),
        # 16 finished threads of a join taken out of an e4m3 cache
        _read("read_join_e4m3", "fp8", 8, 128, 38803, 16),
        # scales from the openings of 16 threads, a small model's heads
        _scales("scales_openings", 2, 1024, 128, False),
        # scales from a calibration batch
        _scales("scales_calibration", 8, 32768, 128, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.random()
    if op < 0.2:
        mode = rng.choice(["bf16", "bf16", "fp8", "fp8", "fp32"])
        head_dim = 128 if mode == "fp8" else rng.choice([64, 128])
        q_heads, kv_heads = rng.choice([(8, 2), (32, 8), (64, 8), (28, 4), (16, 16), (5, 1)])
        most = 8192 * 48 * 128 // ((q_heads + 2 * kv_heads) * head_dim * (2 if mode == "fp32" else 1))
        tokens = _log(rng, 1, most)
        return _write(None, mode, q_heads, kv_heads, head_dim, tokens,
                      rng.choice([0, rng.randrange(tokens)]), rng.random() < 0.8,
                      16 * rng.randint(1, head_dim // 16), rng.choice([1, 1, 2, 3]),
                      rng.random() < 0.4, _log(rng, 1, 1000000))
    if op < 0.35:
        mode = rng.choice(["bf16", "fp8", "fp8", "fp32"])
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        tokens = _log(rng, 1, 38803 * 8 // kv_heads // (2 if mode == "fp32" else 1))
        return _read(None, mode, kv_heads, 128 if mode == "fp8" else rng.choice([64, 128]), tokens,
                     _log(rng, 1, min(tokens, 64)))
    if op < 0.5:
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        return _scales(None, kv_heads, _log(rng, 1, 32768 * 8 // kv_heads), 16 * rng.randint(1, 8),
                       rng.random() < 0.4)
    shape = rng.randrange(1 << 30)
    cap = round(math.exp(rng.uniform(math.log(10), math.log(100))), 2)
    gain = rng.choice([1.0, 1.0, 3.0, 8.0])
    q_heads, kv_heads = rng.choice([(8, 2), (32, 8), (64, 8), (28, 4), (16, 16)])
    if op < 0.7:
        joined = rng.choice([0, 0, _log(rng, 1, 16)])
        tlo = _log(rng, 16, 1024) if joined else 0
        chunks = rng.choice([1, 1, 2, _log(rng, 2, 32)])
        lo = _log(rng, 1, 1024 // chunks)
        case = _attend(None, "prefill", rng.choice(["bf16", "bf16", "fp8"]), q_heads, kv_heads, 128,
                       1, _log(rng, 1, 8192), joined, tlo, _log(rng, tlo, 2048) if joined else 0,
                       chunks, lo, _log(rng, lo, 1024 // chunks), cap, gain, rng.random() < 0.5, shape)
    else:
        mode = rng.choice(["bf16", "bf16", "fp8", "fp32"])
        lo = _log(rng, 1, 4096)
        case = _attend(None, "decode", mode, q_heads, kv_heads,
                       128 if mode == "fp8" else rng.choice([64, 128, 128]), _log(rng, 1, 8),
                       _log(rng, 16, 16384), 0, 0, 0, _log(rng, 1, 48), lo, _log(rng, lo, 8192), cap,
                       gain, rng.random() < 0.5, shape)
    # no larger than the listed cases (the plain form holds every path's keys apart)
    while True:
        w, paths = work(case), case["requests"] * case["leaves"] * case["kv_heads"] * (
            case["prefix"] + case["joined"] * case["threads_hi"] + case["own_hi"])
        if (w["flops"] <= (3e9 if case["mode"] == "fp32" else 6e11) and paths <= 32 * 8 * 24576
                and (case["kind"] == "decode" or paths * case["own_hi"] <= 8 * 1024 * 42000)):
            return case
        key = max(("requests", "leaves", "own_hi", "prefix", "joined"),
                  key=lambda k: case[k] / {"requests": 4, "leaves": 8, "joined": 4}.get(k, 512))
        case[key] = max(1, int(case[key] * 0.7))
        case["own_lo"] = min(case["own_lo"], case["own_hi"])


# ------------------------------------------------------------------ inputs

def _forest(case):
    """(parent, node lengths, leaf or chunk nodes) of an attend case."""
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


def _pool(gen, pages, case):
    """K and V pools of N(0, 1) values, with their scales when they hold e4m3."""
    pools, scales = [], []
    for _ in range(2):
        x = torch.randn((pages, case["kv_heads"], PAGE, case["head_dim"]), generator=gen,
                        device="cuda").to(Q_DTYPE[case["mode"]])
        scale = None
        if case["mode"] == "fp8":
            scale = x.abs().amax(dim=(0, 2, 3)).float() / E4M3_MAX
            x = (x.float() / scale.view(1, -1, 1, 1)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        pools.append(x)
        scales.append(scale)
    return pools[0], pools[1], scales[0], scales[1]


def _tree_inputs(case, seed):
    """An attend case's tree, page table, q and pools."""
    parent, lens, leaves = _forest(case)
    pages = [-(-n // PAGE) for n in lens]
    ptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    ids = np.arange(ptr[-1], dtype=np.int32)
    if case["permuted"]:
        ids = np.random.default_rng(seed).permutation(ids).astype(np.int32)
    gen = _generator(seed)
    queries = sum(lens[n] for n in leaves) if case["kind"] == "prefill" else len(leaves)
    q = (case["gain"] * torch.randn((queries, case["q_heads"], case["head_dim"]), generator=gen,
                                    device="cuda")).to(Q_DTYPE[case["mode"]])
    k_pages, v_pages, k_scale, v_scale = _pool(gen, max(1, int(ptr[-1])), case)
    return dict(parent=parent, lens=lens, leaves=leaves, ptr=ptr, ids=ids, q=q, k_pages=k_pages,
                v_pages=v_pages, k_scale=k_scale, v_scale=v_scale)


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
            dict(slots=slots, q_row=q_row, seen=seen, pick=pick).items()}


def _freqs(case):
    half = case["rotary_dim"] // 2
    return (1e6 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()


def _axes(case):
    """Axis of each frequency: equal contiguous sections."""
    half = case["rotary_dim"] // 2
    return [min(i * case["axes"] // half, case["axes"] - 1) for i in range(half)]


def _token_inputs(case, seed):
    """A write or scales case's rows (views of one projection's output, as a model has them)."""
    gen = _generator(seed)
    h_q, h_kv, d, n = case.get("q_heads", 0), case["kv_heads"], case["head_dim"], case["tokens"]
    qkv = torch.randn((n, (h_q + 2 * h_kv) * d), generator=gen, device="cuda")
    # keys of real models have a few large channels; every head has a magnitude of its own
    qkv *= torch.exp(0.5 * torch.randn(h_q + 2 * h_kv, generator=gen, device="cuda")).repeat_interleave(d)
    qkv = qkv.to(Q_DTYPE[case["mode"]])
    q, k, v = (x.view(n, -1, d) for x in qkv.split([h_q * d, h_kv * d, h_kv * d], dim=1))
    return gen, q, k, v


def _write_inputs(case, seed):
    gen, q, k, v = _token_inputs(case, seed)
    n, live = case["tokens"], case["tokens"] - case["padding"]
    pages = -(-live // PAGE) + 1 + live // (8 * PAGE)
    k_pages, v_pages, k_scale, v_scale = _pool(gen, pages, case)
    if k_scale is not None:     # a little small for the largest values, as scales from other text are
        k_scale, v_scale = (x.float().abs().amax(dim=(0, 2)) * 0.9 / E4M3_MAX for x in (k, v))
    rng = np.random.default_rng(seed)
    table = rng.permutation(pages)[:-(-live // PAGE)]
    slots = np.full(n, -1, dtype=np.int32)
    slots[:live] = (table[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:live]
    # one axis: running positions; several: time runs, the others walk over an image grid
    step = case["first"] + np.arange(n, dtype=np.int64)
    positions = np.stack([step, case["first"] + step // 32 % 32, case["first"] + step % 32][:case["axes"]])
    return dict(q=q if case["with_q"] else None, k=k, v=v, k_pages=k_pages, v_pages=v_pages,
                k_scale=k_scale, v_scale=v_scale, slots=torch.from_numpy(slots).cuda(),
                positions=torch.from_numpy(positions.astype(np.int32)).cuda(), live=live)


def _read_inputs(case, seed):
    gen = _generator(seed)
    n, runs = case["tokens"], case["runs"]
    sizes = [n * (i + 1) // runs - n * i // runs for i in range(runs)]
    pages = sum(-(-s // PAGE) for s in sizes)
    pool = _pool(gen, pages + pages // 8 + 1, case)
    table = np.random.default_rng(seed).permutation(pages + pages // 8 + 1)[:pages]
    slots, at = [], 0
    for s in sizes:
        mine = table[at:at + -(-s // PAGE)]
        slots.append((mine[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:s])
        at += len(mine)
    slots = torch.from_numpy(np.concatenate(slots).astype(np.int32)).cuda()
    return dict(zip(("k_pages", "v_pages", "k_scale", "v_scale"), pool), slots=slots)


def prepare(case, seed):
    op, mode, d = case["op"], case["mode"], case["head_dim"]
    state = {"case": case}
    if op == "attend":
        t = _tree_inputs(case, seed)
        state.update(t, out=torch.empty_like(t["q"]),
                     lse=torch.empty(t["q"].shape[:2], dtype=torch.float32, device="cuda"))
        # what either form keeps between steps: the library its plan, the plain form its index arrays
        if own:
            from paper_2608_24658_gb300.api import Plan
            state["plan"] = Plan(num_q_heads=case["q_heads"], num_kv_heads=case["kv_heads"],
                                 head_dim=d, mode=mode, parent=t["parent"], node_len=t["lens"],
                                 node_page_ptr=t["ptr"], page_ids=t["ids"], leaf_node=t["leaves"],
                                 num_physical_pages=t["k_pages"].shape[0],
                                 prefill=case["kind"] == "prefill", logit_cap=case["cap"])
            state["workspace"] = state["plan"].workspace(t["q"].device)
        else:
            state.update(_index(case, t))
        return state
    if op == "write":
        state.update(_write_inputs(case, seed))
        if case["with_q"]:
            state["q_out"] = torch.empty_like(state["q"], memory_format=torch.contiguous_format)
    elif op == "read":
        state.update(_read_inputs(case, seed))
        shape = (case["tokens"], case["kv_heads"], d)
        state["k"], state["v"] = (torch.empty(shape, dtype=Q_DTYPE[mode], device="cuda") for _ in range(2))
        return state
    else:
        _, _, state["k"], state["v"] = _token_inputs(case, seed)
        state["k_scale"], state["v_scale"] = (torch.empty(case["kv_heads"], device="cuda") for _ in range(2))
    state["inv_freq"] = _freqs(case)
    if op == "write":
        state["axes"] = torch.tensor(_axes(case), device="cuda")
    if own:
        from paper_2608_24658_gb300.api import Rotary
        state["rotary"] = Rotary(state["inv_freq"], axes=_axes(case) if op == "write" else None,
                                 interleaved=case["interleaved"])
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"attend": _attend_own, "write": _write_own, "read": _read_own,
                "scales": _scales_own}[op](state)
    return {"attend": _attend_plain, "write": _write_plain, "read": _read_plain,
            "scales": _scales_plain}[op](state)


def _attend_own(s):
    return s["plan"].decode(s["q"], s["k_pages"], s["v_pages"], out=s["out"], lse=s["lse"],
                            workspace=s["workspace"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _write_own(s):
    from paper_2608_24658_gb300.api import kv_write
    q_out = kv_write(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slots"], q=s["q"],
                     q_out=s.get("q_out"), rotary=s["rotary"], positions=s["positions"],
                     k_scale=s["k_scale"], v_scale=s["v_scale"])
    return {"q": q_out, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _read_own(s):
    from paper_2608_24658_gb300.api import kv_read
    return kv_read(s["k_pages"], s["v_pages"], s["slots"], k=s["k"], v=s["v"],
                   k_scale=s["k_scale"], v_scale=s["v_scale"])


def _scales_own(s):
    from paper_2608_24658_gb300.api import kv_scales
    return kv_scales(s["k"], s["v"], rotary=s["rotary"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def _gathered(pages, scale, slots):
    """Rows [..., H_kv, d] of the slots [...], in 32 bits."""
    raw = pages.view(torch.uint8) if pages.element_size() == 1 else pages
    rows = raw[slots // PAGE, :, slots % PAGE]
    rows = (rows.view(pages.dtype) if pages.element_size() == 1 else rows).float()
    return rows if scale is None else rows * scale.view(-1, 1)


def _attend_plain(s):
    case = s["case"]
    h_q, h_kv, d, cap = case["q_heads"], case["kv_heads"], case["head_dim"], case["cap"]
    g = h_q // h_kv
    n, most = s["q_row"].shape
    k = _gathered(s["k_pages"], s["k_scale"], s["slots"])                    # [n, keys, H_kv, d]
    v = _gathered(s["v_pages"], s["v_scale"], s["slots"])
    q = s["q"][s["q_row"]].float().view(n, most, h_kv, g, d).permute(0, 2, 3, 1, 4)
    x = torch.matmul(q.reshape(n, h_kv, g * most, d), k.permute(0, 2, 3, 1)) / math.sqrt(d)
    x = cap * torch.tanh(x / cap)
    hidden = torch.arange(k.shape[1], device="cuda") >= s["seen"].unsqueeze(-1)   # [n, most, keys]
    x = x.view(n, h_kv, g, most, -1).masked_fill(hidden[:, None, None], -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(n, h_kv, g * most, -1), v.permute(0, 2, 1, 3)).view(n, h_kv, g, most, d) / l
    o = o.permute(0, 3, 1, 2, 4).reshape(n * most, h_q, d)[s["pick"]]
    lse = (m + torch.log(l)).permute(0, 3, 1, 2, 4).reshape(n * most, h_q)[s["pick"]]
    return o.to(s["q"].dtype), lse


def _turned(x, cos, sin, case):
    """x [tokens, heads, d] in 32 bits with its first rotary_dim dims rotated."""
    r = case["rotary_dim"]
    head, rest = x.float().split([r, x.shape[2] - r], dim=2)
    if case["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2), rest], dim=2)
    a, b = head.split(r // 2, dim=2)
    return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], dim=2)


def _stored(x, scale, dtype):
    if scale is None:
        return x.to(dtype)
    return (x / scale.view(-1, 1)).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)


def _write_plain(s):
    case, live = s["case"], s["live"]
    angle = s["positions"][s["axes"]].t().double() * s["inv_freq"].double()  # [tokens, rotary_dim / 2]
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    slots = s["slots"][:live].long()
    page, at = slots // PAGE, slots % PAGE
    for pages, rows, scale in ((s["k_pages"], _turned(s["k"], cos, sin, case), s["k_scale"]),
                               (s["v_pages"], s["v"].float(), s["v_scale"])):
        rows = _stored(rows[:live], scale, pages.dtype)
        if pages.element_size() == 1:
            pages.view(torch.uint8)[page, :, at] = rows.view(torch.uint8)
        else:
            pages[page, :, at] = rows
    q = None if s["q"] is None else _turned(s["q"], cos, sin, case).to(s["q"].dtype)
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _read_plain(s):
    slots = s["slots"].long()
    return tuple(_gathered(pages, scale, slots).to(s["k"].dtype) for pages, scale in
                 ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"])))


def _scales_plain(s):
    case, r = s["case"], s["case"]["rotary_dim"]
    head, rest = s["k"].float().split([r, s["k"].shape[2] - r], dim=2)
    a, b = (head[..., 0::2], head[..., 1::2]) if case["interleaved"] else head.split(r // 2, dim=2)
    k = torch.cat([torch.sqrt(a * a + b * b), rest.abs()], dim=2).amax(dim=(0, 2))
    return k / E4M3_MAX, s["v"].float().abs().amax(dim=(0, 2)) / E4M3_MAX


# ------------------------------------------------------------------ work

def work(case):
    h_kv, d, mode = case["kv_heads"], case["head_dim"], case["mode"]
    qb, kvb = Q_BYTES[mode], KV_BYTES[mode]
    n = case.get("tokens", 0)
    if case["op"] == "write":
        heads = h_kv + (case["q_heads"] if case["with_q"] else 0)
        live = n - case["padding"]
        return {"bytes": ((heads - h_kv) * n * 2 * qb + live * 2 * h_kv * (qb + kvb)) * d
                + n * 4 * (1 + case["axes"]),
                "flops": n * heads * case["rotary_dim"] * 3}
    if case["op"] == "read":
        return {"bytes": 2 * n * h_kv * d * (qb + kvb) + 4 * n, "flops": 2 * n * h_kv * d}
    if case["op"] == "scales":
        return {"bytes": 2 * n * h_kv * d * qb + 8 * h_kv, "flops": 4 * n * h_kv * d}
    parent, lens, leaves = _forest(case)
    under = [0] * len(parent)
    for i in leaves:
        under[i] = lens[i] if case["kind"] == "prefill" else 1
    queries = sum(under)
    for i in range(len(parent) - 1, 0, -1):
        if parent[i] >= 0:
            under[parent[i]] += under[i]
    mine = set(leaves) if case["kind"] == "prefill" else set()    # causal in the chunk itself
    keys = sum(lens[i] * (lens[i] + 1) // 2 if i in mine else lens[i] * under[i]
               for i in range(len(parent)))
    return {"bytes": sum(lens) * 2 * h_kv * d * kvb + queries * case["q_heads"] * (2 * d * qb + 4),
            "flops": keys * case["q_heads"] * 4 * d}


# ------------------------------------------------------------------ in 64 bits

def _wide(x):
    return x.to(torch.float32).to(torch.float64)


def _exact_attend(case, seed):
    t = _tree_inputs(case, seed)
    h_q, h_kv, d, cap = case["q_heads"], case["kv_heads"], case["head_dim"], case["cap"]
    g = h_q // h_kv
    out = torch.empty(t["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(t["q"].shape[:2], dtype=torch.float64, device="cuda")
    nodes = {}

    def node(n):
        if n not in nodes:
            ids = torch.from_numpy(t["ids"][t["ptr"][n]:t["ptr"][n + 1]].astype(np.int64)).cuda()
            kv = []
            for pages, scale in ((t["k_pages"], t["k_scale"]), (t["v_pages"], t["v_scale"])):
                x = pages.view(torch.uint8)[ids].view(pages.dtype) if pages.element_size() == 1 else pages[ids]
                x = _wide(x).transpose(0, 1).reshape(h_kv, -1, d)[:, :t["lens"][n]]
                kv.append(x if scale is None else x * _wide(scale).view(-1, 1, 1))
            nodes[n] = kv
        return nodes[n]

    row = 0
    for leaf in t["leaves"]:
        path = _path(t, leaf)
        k, v = (torch.cat([node(n)[i] for n in path], dim=1) for i in range(2))
        nodes.pop(leaf)
        for n in [n for n in nodes if n not in path]:
            nodes.pop(n)
        queries = t["lens"][leaf] if case["kind"] == "prefill" else 1
        total = k.shape[1]
        for t0 in range(0, queries, 128):
            t1 = min(queries, t0 + 128)
            for h in range(h_kv):
                q = _wide(t["q"][row + t0:row + t1, h * g:(h + 1) * g])            # [rows, g, d]
                s = cap * torch.tanh(torch.einsum("tgd,kd->gtk", q, k[h]) / (math.sqrt(d) * cap))
                if queries > 1:
                    last = total - queries + torch.arange(t0, t1, device="cuda")
                    s.masked_fill_(torch.arange(total, device="cuda") > last[:, None], -math.inf)
                z = torch.logsumexp(s, dim=-1)
                lse[row + t0:row + t1, h * g:(h + 1) * g] = z.t()
                out[row + t0:row + t1, h * g:(h + 1) * g] = torch.einsum(
                    "gtk,kd->tgd", torch.exp(s - z.unsqueeze(-1)), v[h])
        row += queries
    return out, lse


def _exact_write(case, seed):
    s = _write_inputs(case, seed)
    r, n = case["rotary_dim"], case["tokens"]
    positions, freqs, axes = s["positions"].double(), _freqs(case).double(), _axes(case)
    turn = torch.polar(torch.ones(n, len(axes), dtype=torch.float64, device="cuda"),
                       torch.stack([positions[a] * f for a, f in zip(axes, freqs)], dim=1)).unsqueeze(1)

    def rotated(x):
        x = _wide(x).clone()
        first, second = (x[..., 0:r:2], x[..., 1:r:2]) if case["interleaved"] else (
            x[..., :r // 2], x[..., r // 2:r])
        z = torch.complex(first, second) * turn
        first.copy_(z.real), second.copy_(z.imag)
        return x

    result = {"q": None if s["q"] is None else rotated(s["q"])}
    slots = s["slots"][s["slots"] >= 0].long()
    for name, rows in (("k", rotated(s["k"])), ("v", _wide(s["v"]))):
        pages, scale = _wide(s[name + "_pages"]), s[name + "_scale"]
        if scale is not None:
            rows = (rows / _wide(scale).view(-1, 1)).clamp(-E4M3_MAX, E4M3_MAX)
        pages[slots // PAGE, :, slots % PAGE] = rows[:len(slots)]
        result[name + "_pages"] = pages
    return result


def _exact_read(case, seed):
    s = _read_inputs(case, seed)
    got = []
    for pages, scale in ((s["k_pages"], s["k_scale"]), (s["v_pages"], s["v_scale"])):
        rows = _wide(pages).transpose(1, 2).reshape(-1, case["kv_heads"], case["head_dim"])[s["slots"].long()]
        got.append(rows if scale is None else rows * _wide(scale).view(-1, 1))
    return tuple(got)


def _exact_scales(case, seed):
    _, _, k, v = _token_inputs(case, seed)
    r, k, v = case["rotary_dim"], _wide(k), _wide(v)
    pairs = k[..., :r].unflatten(-1, (r // 2, 2) if case["interleaved"] else (2, r // 2))
    most = torch.linalg.vector_norm(pairs, dim=-1 if case["interleaved"] else -2).amax(dim=(0, 2))
    if r < case["head_dim"]:
        most = torch.maximum(most, k[..., r:].abs().amax(dim=(0, 2)))
    return most / E4M3_MAX, v.abs().amax(dim=(0, 2)) / E4M3_MAX


def exact(case, seed):
    return {"attend": _exact_attend, "write": _exact_write, "read": _exact_read,
            "scales": _exact_scales}[case["op"]](case, seed)
