"""parason_plan_fork cuts the suffix pass's pieces as the plan does: in 4 bits whole stages of
two pages but for a node's last piece."""
import numpy as np
import pytest

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import Plan
from tests.plan_cover import coverage, definition


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def pieces(plan, tree, first):
    """(pages, whether they end their node) of items from `first` on."""
    ptr = np.asarray(tree.node_page_ptr)
    got = []
    for it in plan.export(_lib.TABLE_ITEMS)[first:]:
        pos, pages = int(it[0]), int(it[1])
        node = int(np.searchsorted(ptr, pos, side="right")) - 1
        assert pos + pages <= ptr[node + 1]
        got.append((pages, pos + pages == ptr[node + 1]))
    return got


@pytest.mark.parametrize("mode", ["fp4", "bf16"])
@pytest.mark.parametrize("tokens", [33, 300, 900, 2500, 5000, 9000])
@pytest.mark.parametrize("sms", [3, 8, 152])
def test_pieces_of_a_fork(tokens, sms, mode):
    tree = W.build_tree("pieces", [-1, 0, 0, 0], [2 * tokens, tokens, tokens + 40, 17], [1, 2, 3], num_q_heads=8,
                        num_kv_heads=2, head_dim=128, mode=mode, values=False, extra_pages=tokens // 4 + 40,
                        permute_pages=False)
    pool = W.free_pages(tree)
    with Plan.for_tree(tree, host_only=True, num_sms=sms) as plan:
        first = plan.info()["num_items"]
        lens = [tokens, 3 * tokens // 2, 5]
        tree, pages = W.fork_branch(tree, 1, lens, pool)
        plan.fork(1, lens, pages)
        assert coverage(plan) == definition(tree)
        new = pieces(plan, tree, first)
    assert new
    if mode == "fp4":
        assert all(n % 2 == 0 for n, last in new if not last)
