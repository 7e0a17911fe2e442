"""kv_slots with all its arrays side by side in one buffer, lengths and outputs between the table's
rows: taken, and right; over one another they are refused."""
import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import build
from paper_2608_24658_gb300.api import ParasonError, kv_slots
from tests import slots_ref as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    torch.cuda.init()


SEQS, WIDTH, ROWS = 6, 4, 60
SIZES = dict(held=SEQS, added=SEQS, first=SEQS, free_pages=20, free_used=1, slots=ROWS, positions=ROWS,
             token_ptr=SEQS + 1, lens_out=SEQS, used_out=1)


def arrays(order):
    """The arrays in `order`, each in the gaps behind the table's rows as far as they reach, then behind it."""
    stride = WIDTH + 70
    buffer = torch.full((SEQS * stride + 400,), -9, dtype=torch.int32, device="cuda")
    got, row, at = {"page_table": buffer[:SEQS * stride].view(SEQS, stride)[:, :WIDTH]}, 0, WIDTH
    for name in order:
        n = SIZES[name]
        if row < SEQS and at + n > stride:
            row, at = row + 1, WIDTH
        got[name] = buffer[row * stride + at:row * stride + at + n]
        at += n
    return buffer, got


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("in_place", [False, True])
def test_neighbours(seed, in_place):
    rng = np.random.default_rng(seed)
    order = [str(n) for n in rng.permutation(sorted(SIZES))]
    buffer, a = arrays(order)
    held, added, first = rng.integers(0, 30, SEQS), rng.integers(0, 12, SEQS), rng.integers(0, 99, SEQS)
    free, table = 100 + rng.permutation(20), rng.permutation(SEQS * WIDTH).reshape(SEQS, WIDTH)
    for name, x in (("held", held), ("added", added), ("first", first), ("free_pages", free), ("free_used", [2]),
                    ("page_table", table)):
        a[name].copy_(torch.from_numpy(np.asarray(x, np.int32)))
    if in_place:
        a["lens_out"], a["used_out"] = a["held"], a["free_used"]
    kw = {n: t for n, t in a.items() if n not in ("page_table", "held")}
    kv_slots(a["page_table"], a["held"], **kw)
    want = S.slots(table, held, added, ROWS, first, free, 2)
    for name, w in zip(("slots", "positions", "token_ptr", "lens_out", "used_out", "page_table"), want):
        assert np.array_equal(a[name].cpu().numpy().squeeze(), np.asarray(w).squeeze()), name
    kept = buffer.clone()
    for out, over in (("lens_out", "added"), ("slots", "positions"), ("token_ptr", "held"), ("used_out", "first")):
        bad = dict(kw)
        bad[out] = a[over][:SIZES[out]]
        if len(bad[out]) == SIZES[out]:
            with pytest.raises(ParasonError):
                kv_slots(a["page_table"], a["held"], **bad)
    assert torch.equal(buffer, kept)
