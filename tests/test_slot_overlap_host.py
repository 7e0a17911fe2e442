"""kv_slots refuses outputs that lie over what it reads or over one another (lens_out and used_out
may be held and free_used): its CTAs read lengths, lists and table while others write.  Nothing
here is launched."""
import ctypes

import pytest

from paper_2608_24658_gb300 import _lib, build

# three sequences of five pages, nine rows, a list of four: each array in a place of its own
AT = {name: (1 << 20) + 4096 * i for i, name in enumerate(
    ("held", "added", "first", "page_table", "free_pages", "free_used", "slots", "positions", "token_ptr", "held_out",
     "used_out"))}
SIZE = dict(held=3, added=3, first=3, page_table=15, free_pages=4, free_used=1, slots=9, positions=9, token_ptr=4,
            held_out=3, used_out=1)
OUTPUTS = ("slots", "positions", "token_ptr", "held_out", "used_out", "page_table")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def call(lib, **kw):
    f = dict(AT, num_seqs=3, num_rows=9, table_stride=5, table_pages=5, num_free=4)
    f.update(kw)
    return lib.parason_kv_slots(ctypes.byref(_lib.SlotMap(**f)), None)


@pytest.mark.parametrize("out", OUTPUTS)
@pytest.mark.parametrize("other", sorted(AT))
def test_overlaps(lib, out, other):
    if out == other:
        return
    allowed = {("held_out", "held"), ("used_out", "free_used")}
    if (out, other) not in allowed:
        assert call(lib, **{out: AT[other]}) == _lib.EINVAL
        assert call(lib, **{out: AT[other] + 4 * (SIZE[other] - 1)}) == _lib.EINVAL
    if SIZE[out] > 1:
        assert call(lib, **{out: AT[other] - 4 * (SIZE[out] - 1)}) == _lib.EINVAL


@pytest.mark.parametrize("out,at", [("slots", 0), ("slots", -5), ("positions", 33), ("token_ptr", 38), ("held_out", 84),
                                    ("used_out", 44), ("used_out", 80)])
def test_rows_that_lie_apart(lib, out, at):
    """Rows of 5 pages, 40 entries apart: inside one of them, across its start or end."""
    assert any(40 * r - SIZE[out] < at < 40 * r + 5 for r in range(3))
    assert call(lib, table_stride=40, **{out: AT["page_table"] + 4 * at}) == _lib.EINVAL


@pytest.mark.parametrize("bad", [
    dict(num_seqs=-1), dict(num_rows=-1), dict(table_pages=-1), dict(num_free=-1), dict(held=None),
    dict(page_table=None), dict(table_stride=4), dict(table_stride=-5), dict(slots=None), dict(slots=AT["slots"] + 2),
    dict(free_pages=None), dict(free_pages=None, num_free=0), dict(positions=AT["positions"] + 1)])
def test_refusals_of_arrays_apart(lib, bad):
    assert call(lib, **bad) == _lib.EINVAL


def test_too_large_first(lib):
    assert call(lib, num_seqs=16385, held_out=AT["added"]) == _lib.EUNSUPPORTED
    assert call(lib, num_rows=2 ** 31 - 1) == _lib.EUNSUPPORTED
