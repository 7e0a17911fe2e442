"""kv_slots at its most sequences with lengths and list advanced in place: one cluster, whose CTAs
hold all lengths each; and a step after a step of it, captured."""
import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import kv_slots
from tests import slots_ref as S
from tests import test_kv_slots_gpu as slots

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


@pytest.mark.parametrize("seqs", [16384, 12001, 4096])
@pytest.mark.parametrize("most", [1, 3, 40])
def test_in_place(seqs, most):
    rng = np.random.default_rng(seqs + most)
    held, added = rng.integers(0, 40, seqs), rng.integers(0, most + 1, seqs)
    slots.check(held, added, int(added.sum()) + 3, free=rng.permutation(int(added.sum()) // 16 + seqs), in_place=True)


def test_replayed_in_place():
    rng = np.random.default_rng(3)
    seqs = 16384
    held, table = rng.integers(0, 30, seqs), np.full((seqs, 4), -1)
    free = rng.permutation(4 * seqs)
    for r in range(seqs):
        table[r, :-(-held[r] // 16)] = 10 ** 6 + 4 * r + np.arange(-(-held[r] // 16))
    d = [slots.dev(x) for x in (table, held, free, [0])]
    out = [torch.empty(seqs, dtype=torch.int32, device="cuda") for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv_slots(d[0], d[1], free_pages=d[2], free_used=d[3], slots=out[0], positions=out[1], lens_out=d[1], used_out=d[3])
    used = 0
    for _ in range(3):
        graph.replay()
        want = S.slots(table, held, None, seqs, None, free, used)
        held, used, table = want[3], want[4], want[5]
        for got, w in ((out[0], want[0]), (out[1], want[1]), (d[1], held), (d[0], table)):
            assert np.array_equal(got.cpu().numpy(), w)
        assert int(d[3]) == used
