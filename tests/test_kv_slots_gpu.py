"""kv_slots against a loop, at the lengths, tables and lists where it can go wrong."""
import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import kv_slots
from tests import slots_ref as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def check(held, added, rows, width=None, first=None, free=None, used=0, table=None, stride=0, in_place=False, seed=0):
    rng = np.random.default_rng(seed)
    held = np.asarray(held, np.int64)
    had = -(-np.maximum(held, 0) // 16)
    need = -(-np.maximum(held + (1 if added is None else np.maximum(added, 0)), 0) // 16)
    width = int(max(need.max(initial=0), had.max(initial=0))) + 1 if width is None else width
    if table is None:
        table = rng.permutation(len(held) * width).reshape(len(held), width)
        if free is not None:
            for r in range(len(held)):
                table[r, had[r]:] = -1
    full = torch.full((len(held), width + stride), -7, dtype=torch.int32, device="cuda")
    t = full[:, :width]
    t.copy_(dev(table))
    d_held, d_used = dev(held), dev([used]) if free is not None else None
    outs = dict(token_ptr=torch.empty(len(held) + 1, dtype=torch.int32, device="cuda"),
                lens_out=d_held if in_place else torch.empty_like(d_held))
    if free is not None:
        outs["used_out"] = d_used if in_place else torch.empty_like(d_used)
    slots, pos = kv_slots(t, d_held, dev(added), rows, first=dev(first), free_pages=dev(free), free_used=d_used, **outs)
    want = S.slots(table, held, added, rows, first, free, used)
    for got, w in ((slots, want[0]), (pos, want[1]), (outs["token_ptr"], want[2]), (outs["lens_out"], want[3]),
                   (t, want[5])):
        assert np.array_equal(got.cpu().numpy(), w)
    if free is not None:
        assert int(outs["used_out"]) == want[4]
    assert (full[:, width:] == -7).all()


@pytest.mark.parametrize("seqs", [1, 2, 31, 33, 300, 1025, 2500])
@pytest.mark.parametrize("listed", [False, True])
def test_a_step(seqs, listed):
    rng = np.random.default_rng(seqs)
    held = rng.integers(0, 200, seqs)
    free = 5000 + rng.permutation(seqs + 9) if listed else None
    check(held, None, seqs, first=rng.integers(0, 5000, seqs), free=free, used=4 if listed else 0)


@pytest.mark.parametrize("seqs,most", [(1, 1), (1, 40), (1, 30000), (3, 5000), (70, 300), (1100, 60)])
@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("spare", [0, 3, 1000])
def test_ragged(seqs, most, listed, spare):
    rng = np.random.default_rng(seqs + most)
    held, added = rng.integers(0, 100, seqs), rng.integers(0, most + 1, seqs)
    free = 10 ** 6 + rng.permutation(int(added.sum()) // 16 + 2 * seqs) if listed else None
    check(held, added, int(added.sum()) + spare, first=rng.integers(0, 9, seqs), free=free, stride=5)


@pytest.mark.parametrize("lengths", [([0, 15, 16, 17, 31, 32], [16, 1, 1, 15, 33, 0]), ([0, 0, 0], [0, 0, 0]),
                                     ([5], [0]), ([16, 0, 16], [0, 5, 0])])
def test_edges(lengths):
    held, added = (np.array(x) for x in lengths)
    for free in (None, np.arange(100, 120)):
        check(held, added, int(added.sum()) + 2, free=free)
        check(held, added, int(added.sum()), free=free, in_place=True)


@pytest.mark.parametrize("free,used", [(1, 0), (5, 0), (5, 3), (5, 5), (5, 900), (12, -4)])
def test_a_list_that_runs_out(free, used):
    held, added = np.array([3, 16, 30, 0, 40]), np.array([20, 50, 2, 33, 7])
    check(held, added, 112, free=np.arange(50, 50 + free), used=used)


def test_narrow_tables():
    held, added = np.array([3, 16, 90, 0]), np.array([60, 50, 5, 100])
    for free in (None, np.arange(50, 90)):
        check(held, added, 215, width=3, free=free, table=np.arange(12).reshape(4, 3))
    check(held, added, 215, width=0, table=np.empty((4, 0), np.int64))


@pytest.mark.parametrize("rows", [0, 1, 30, 31, 79, 109])
def test_fewer_rows_than_tokens(rows):
    held, added = np.array([3, 16, 90, 0]), np.array([30, 50, 5, 25])
    for free in (None, np.arange(50, 90)):
        check(held, added, rows, free=free)


def test_tables_with_holes_and_wild_lengths():
    table = np.array([[4, -1, 2 ** 31 - 1], [(2 ** 31 - 1) // 16, 3, -2 ** 31]])
    check(np.array([0, 0]), np.array([48, 48]), 96, width=3, table=table)
    check(np.array([-5, 7]), np.array([20, -3]), 20, width=3, table=np.arange(6).reshape(2, 3))
    check(np.array([2 ** 31 - 5, 3]), np.array([100, 9]), 30, width=2, table=np.arange(4).reshape(2, 2))
    check(np.array([0, 0, 0]), np.array([2 ** 31 - 1] * 3), 50, width=5, free=np.arange(9), table=np.full((3, 5), -1))


def test_most_sequences():
    rng = np.random.default_rng(1)
    held, added = rng.integers(0, 40, 16384), rng.integers(0, 4, 16384)
    check(held, added, int(added.sum()) + 1, free=rng.permutation(20000))


def test_no_sequences_and_defaults():
    slots, pos = kv_slots(torch.empty((0, 4), dtype=torch.int32, device="cuda"),
                          torch.empty(0, dtype=torch.int32, device="cuda"), tokens=9)
    assert (slots == -1).all() and (pos == 0).all()
    table = torch.tensor([[7, 9]], dtype=torch.int32, device="cuda")
    slots, pos = kv_slots(table, torch.tensor([17], dtype=torch.int32, device="cuda"))
    assert slots.tolist() == [145] and pos.tolist() == [17]


def test_unaligned_outputs():
    rng = np.random.default_rng(2)
    held, added = rng.integers(0, 40, 50), rng.integers(0, 30, 50)
    n = int(added.sum())
    table = rng.permutation(50 * 6).reshape(50, 6)
    buffer = torch.full((2, n + 9), -9, dtype=torch.int32, device="cuda")
    kv_slots(dev(table), dev(held), dev(added), slots=buffer[0, 1:n + 1], positions=buffer[1, 3:n + 3])
    want = S.slots(table, held, added, n)
    assert np.array_equal(buffer[0, 1:n + 1].cpu(), want[0]) and np.array_equal(buffer[1, 3:n + 3].cpu(), want[1])
    assert (buffer[0, 0] == -9) and (buffer[0, n + 1:] == -9).all() and (buffer[1, n + 3:] == -9).all()


def test_captured_steps_advance_in_place():
    held, used = dev([14, 0, 31]), dev([0])
    table = dev(np.array([[1, -1, -1], [-1, -1, -1], [2, 3, -1]]))
    free = dev([10, 11, 12, 13])
    slots, pos = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv_slots(table, held, free_pages=free, free_used=used, slots=slots, positions=pos, lens_out=held, used_out=used)
    seen = []
    for _ in range(3):
        graph.replay()
        seen.append((slots.tolist(), pos.tolist()))
    assert seen == [([30, 160, 63], [14, 0, 31]), ([31, 161, 176], [15, 1, 32]), ([192, 162, 177], [16, 2, 33])]
    assert held.tolist() == [17, 3, 34] and used.tolist() == [3]
    assert table.tolist() == [[1, 12, -1], [10, -1, -1], [2, 3, 11]]


def test_what_is_refused():
    i = dict(dtype=torch.int32, device="cuda")
    table, held, free = torch.zeros((3, 4), **i), torch.zeros(3, **i), torch.zeros(5, **i)
    for bad in (dict(page_table=table.long()), dict(page_table=table[0]), dict(page_table=table.t()),
                dict(held=held[:2]), dict(held=held.long()), dict(added=held), dict(added=held[:2], tokens=3),
                dict(first=torch.zeros(6, **i)[::2]), dict(free_used=torch.zeros(1, **i)),
                dict(free_pages=free, free_used=torch.zeros(2, **i)), dict(free_pages=free[:0]),
                dict(used_out=torch.zeros(1, **i)), dict(slots=torch.zeros((3, 1), **i)),
                dict(slots=torch.zeros(3, **i), tokens=4), dict(tokens=-1), dict(token_ptr=held),
                dict(slots=torch.zeros(3, **i), positions=torch.zeros(4, **i)), dict(lens_out=torch.zeros(4, **i))):
        with pytest.raises(ValueError):
            kv_slots(**dict(dict(page_table=table, held=held), **bad))
