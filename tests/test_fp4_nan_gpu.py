"""4-bit KV: a NaN score makes its row's out and lse NaN, in every tile, merge and epilogue; a wait
that runs out ends a decode or a prefill with an error, and the next one is right."""
import math

import pytest
import torch

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300.api import ParasonError, Plan
from tests import fp4_ref as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def run(t, cap, prefill=False):
    with Plan.for_tree(t, prefill=prefill, logit_cap=cap) as plan:
        out, lse = plan.decode_tree(t)
        plan.check()
        return out, lse


def check(t, cap, out, lse, rows, prefill=False):
    """NaN in all of `rows` rows of heads, the others as near as ever (the bounds of fp4_ref.check)."""
    ref, z, mean, size, tiny = F.attend(t, prefill, cap)
    lost = z.isnan()
    assert int(lost.sum()) == rows
    assert out[lost].isnan().all(), f"{int((~out[lost].isnan()).sum())} finite elements"
    assert lse[lost].isnan().all(), lse[lost][~lse[lost].isnan()][:4].tolist()
    score = 2.0 ** -16 * size + 2.0 ** -19 * cap
    live = ~lost & (z > -math.inf)
    assert ((lse.double() - z).abs() <= score + 2.0 ** -20 * (1.0 + z.abs()))[live].all()
    p = 2.0 ** -11 + 2.0 ** -15 + 2 * score.unsqueeze(-1)
    most = 2.0 ** -8 * ref.abs() + (1 + 2.0 ** -8) * (p * mean + 2.0 ** -25 * tiny)
    assert ((out.double() - ref).abs() <= most)[live].all()
    empty = z == -math.inf
    assert (lse[empty] == -math.inf).all() and (out[empty] == 0).all()


def spoil(t, node, tokens, head, block=3):
    """One block's scale of these keys of a node becomes NaN."""
    scales = F.split(t.k_pages)[1]
    for i in tokens:
        scales[int(t.page_ids[int(t.node_page_ptr[node]) + i // 16]), head, i % 16, block] = F.NAN_SCALE


CAPS = [0.0, 50.0, 90.0]

# (branches, heads, prefix, own): tiles of 4, 12 and 16 rows, a shared prefix's of several row tiles, no prefix
DECODES = {"four": (6, (8, 2), 300, 40), "twelve": (2, (24, 2), 0, 70), "sixteen": (3, (32, 2), 40, 33),
           "shared": (40, (16, 2), 130, 20), "many": (150, (32, 4), 130, 20), "short": (6, (8, 2), 0, 9),
           "alone": (1, (4, 2), 0, 2000)}


@pytest.mark.parametrize("case", sorted(DECODES))
@pytest.mark.parametrize("cap", CAPS)
def test_decode(case, cap):
    """One branch's last key; every key of a branch's path; a branch's first stage; a query."""
    leaves, (h_q, h_kv), prefix, own = DECODES[case]
    lens = [prefix] + [own + i % 7 for i in range(leaves)]

    def tree():
        return F.tree_of([-1] + [0] * leaves, lens, list(range(1, leaves + 1)), h_q, h_kv, seed=3)
    group, last = h_q // h_kv, leaves
    one, whole, first, query = (tree() for _ in range(4))
    spoil(one, last, [lens[last] - 1], 1)
    check(one, cap, *run(one, cap), group)
    spoil(whole, 0, range(prefix), 1)
    spoil(whole, last, range(lens[last]), 1)
    check(whole, cap, *run(whole, cap), group * (leaves if prefix else 1))
    spoil(first, 1, range(min(32, lens[1])), 0, 7)
    check(first, cap, *run(first, cap), group)
    query.q[leaves // 2, 1, 77] = math.nan
    check(query, cap, *run(query, cap), 1)


PREFILLS = {"direct": ([-1, 0, 0], [60, 64, 70], [1, 2]), "merged": ([-1, 0, 0], [9000, 130, 30], [1, 2]),
            "root": ([-1], [90], [0])}


@pytest.mark.parametrize("case", sorted(PREFILLS))
@pytest.mark.parametrize("cap", CAPS)
def test_prefill(case, cap):
    parent, lens, chunks = PREFILLS[case]

    def tree():
        return F.tree_of(parent, lens, chunks, 8, 2, seed=4, prefill=True)
    one, whole, query = (tree() for _ in range(3))
    spoil(one, chunks[-1], [17], 1)
    check(one, cap, *run(one, cap, True), (lens[chunks[-1]] - 17) * 4, True)
    for n in range(len(lens)):
        spoil(whole, n, range(lens[n]), 0)
    check(whole, cap, *run(whole, cap, True), whole.q.shape[0] * 4, True)
    query.q[5, 2, 11] = math.nan
    check(query, cap, *run(query, cap, True), 1, True)


@pytest.mark.parametrize("case", ["suffix", "prefix", "prefill"])
def test_a_wait_that_runs_out(case):
    """The first load left out: ETIMEOUT after 2 ms, and the plan goes on."""
    t = {"suffix": lambda: F.tree_of([-1, 0, 0], [100, 300, 17], [1, 2], 8, 2, seed=5),
         "prefix": lambda: F.tree_of([-1] + [0] * 12, [1500] + [40] * 12, list(range(1, 13)), 16, 2, seed=5),
         "prefill": lambda: F.tree_of([-1, 0, 0], [300, 70, 130], [1, 2], 8, 2, seed=5, prefill=True)}[case]()
    with Plan.for_tree(t, prefill=case == "prefill") as plan:
        info = plan.info()
        assert (info["num_wide_items"] > 0) == (case != "suffix")
        plan.set_debug(_lib.DEBUG_SKIP_FIRST_LOAD, wait_limit_ns=2_000_000)
        plan.decode_tree(t)
        with pytest.raises(ParasonError) as e:
            plan.check()
        assert e.value.status == _lib.ETIMEOUT
        plan.set_debug(0, wait_limit_ns=2_000_000_000)
        for _ in range(2):
            out, lse = plan.decode_tree(t)
        plan.check()
    F.check(t, out, lse, case == "prefill")
