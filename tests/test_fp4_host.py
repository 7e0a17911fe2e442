"""Refusals of the 4-bit mode, of normed writes and of kv_slots through the C ABI, and
4-bit plans, where no GPU is needed: nothing here is launched."""
import ctypes

import pytest

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300 import workloads as W
from paper_2608_24658_gb300.api import ParasonError, Plan
from tests.test_plan import verify_plan

A = 1 << 20          # an address that nothing reads


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def _cfg(mode="fp4", **kw):
    f = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, mode=_lib.MODES[mode], sm_scale=0.0)
    f.update(kw)
    return _lib.AttnConfig(**f)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rows(data=A, ts=1024, hs=128):
    return _lib.Rows(data, ts, hs)


def _norm(**kw):
    f = dict(q_weight=A, k_weight=A, q_head_stride=0, k_head_stride=0, eps=1e-6, weight_offset=0.0)
    f.update(kw)
    return _lib.HeadNormDesc(**f)


def _write(lib, cfg=None, n=4, q=None, k=_rows(), v=_rows(), norm=None, slots=A, ks=A, vs=A, q_out=None, kp=A,
           vp=A + 64, pages=10):
    return lib.parason_kv_write_norm(_ref(cfg or _cfg()), n, _ref(q), _ref(k), _ref(v), _ref(norm), None, slots, ks,
                                     vs, q_out, kp, vp, pages, None)


@pytest.mark.parametrize("bad", [dict(ks=None), dict(vs=None), dict(ks=A + 2), dict(kp=None), dict(vp=A + 8),
                                 dict(kp=A + 64), dict(slots=None), dict(k=None), dict(v=_rows(ts=100)),
                                 dict(q=_rows()), dict(q=_rows(), q_out=A + 4), dict(n=-1), dict(pages=-1)])
def test_write_refusals(lib, bad):
    assert _write(lib, **bad) == _lib.EINVAL
    assert _write(lib, norm=_norm(), **bad) == _lib.EINVAL


@pytest.mark.parametrize("bad", [dict(q_weight=None, k_weight=None), dict(q_weight=A + 8), dict(k_weight=A + 2),
                                 dict(q_head_stride=-128), dict(k_head_stride=2), dict(eps=0.0), dict(eps=-1.0),
                                 dict(eps=1e-39), dict(eps=float("nan")), dict(eps=float("inf")),
                                 dict(weight_offset=float("inf")), dict(weight_offset=float("nan"))])
@pytest.mark.parametrize("mode", ["bf16", "fp32", "fp8", "fp4"])
def test_norm_refusals(lib, bad, mode):
    assert _write(lib, _cfg(mode), norm=_norm(**bad)) == _lib.EINVAL
    # checked for an empty batch too, which launches nothing
    assert _write(lib, _cfg(mode), n=0, norm=_norm(**bad)) == _lib.EINVAL
    assert _write(lib, _cfg(mode), n=0, norm=_norm(), k=None, v=None, slots=None) == _lib.OK


def test_shapes_without_a_kernel(lib):
    small = _cfg(head_dim=64)
    assert _write(lib, small) == _lib.EUNSUPPORTED
    rows = _rows()
    assert lib.parason_kv_read(_ref(small), 4, A, A, A + 64, 10, A, A, _ref(rows), _ref(_rows(A + 64)),
                               None) == _lib.EUNSUPPORTED
    assert lib.parason_kv_scales(_ref(small), 4, _ref(rows), _ref(rows), None, None, 0, A, A, None) == _lib.EUNSUPPORTED
    assert lib.parason_kv_read(_ref(_cfg()), 4, A, A, A + 64, 10, None, A, _ref(rows), _ref(_rows(A + 64)),
                               None) == _lib.EINVAL


def _map(**kw):
    f = dict(num_seqs=3, num_rows=9, held=A, added=A, first=None, page_table=A, table_stride=5, table_pages=5,
             num_free=4, free_pages=A, free_used=None, slots=A, positions=A + 64, token_ptr=None, held_out=None,
             used_out=None)
    f.update(kw)
    return _lib.SlotMap(**f)


@pytest.mark.parametrize("bad", [
    dict(num_seqs=-1), dict(num_rows=-1), dict(table_pages=-1), dict(num_free=-1), dict(held=None),
    dict(page_table=None), dict(table_stride=4), dict(table_stride=-5), dict(slots=None), dict(slots=A + 2),
    dict(positions=A + 1), dict(positions=A), dict(held=A + 3), dict(added=A + 2), dict(first=A + 2),
    dict(page_table=A + 1), dict(free_pages=A + 1), dict(free_used=A + 2), dict(token_ptr=A + 2),
    dict(held_out=A + 2), dict(used_out=A + 1), dict(free_pages=None), dict(free_pages=None, num_free=0, free_used=A),
    dict(free_pages=None, num_free=0, used_out=A)])
def test_slot_map_refusals(lib, bad):
    assert lib.parason_kv_slots(_ref(_map(**bad)), None) == _lib.EINVAL


def test_slot_maps_too_large(lib):
    assert lib.parason_kv_slots(None, None) == _lib.EINVAL
    assert lib.parason_kv_slots(_ref(_map(num_seqs=16385)), None) == _lib.EUNSUPPORTED
    assert lib.parason_kv_slots(_ref(_map(num_rows=2 ** 31 - 1)), None) == _lib.EUNSUPPORTED


def test_plans(lib):
    """A 4-bit plan takes head_dim 128, decode and prefill, and every update a plan has."""
    tree = W.figure3_tree(d=128, values=False)
    tree.mode = "fp4"
    with Plan.for_tree(tree, host_only=True, logit_cap=30.0) as plan:
        info = plan.info()
        assert info["num_items"] > 0 and info["unique_tokens"] == tree.unique_tokens()
    parent, lens = [-1, 0, 0], [40, 20, 33]
    ptr, ids, pages = W.assign_pages(lens)
    kw = dict(num_q_heads=8, num_kv_heads=2, parent=parent, node_len=lens, node_page_ptr=ptr, page_ids=ids,
              leaf_node=[1, 2], num_physical_pages=pages + 8, host_only=True, mode="fp4")
    with Plan(head_dim=128, **kw) as plan:
        plan.append()
        assert plan.fork(0, [3, 0], [[pages], []]) == [0, 2]
    with Plan(head_dim=128, prefill=True, **kw) as plan:
        assert plan.num_leaves == 53
    for prefill in (False, True):
        with pytest.raises(ParasonError) as e:
            Plan(head_dim=64, prefill=prefill, **kw)
        assert e.value.status == _lib.EUNSUPPORTED


@pytest.mark.parametrize("prefix, branches, tokens, h_q, sms", [
    (0, 1, 1, 8, 152), (17, 3, 33, 8, 152), (256, 4, 64, 64, 152), (512, 16, 1500, 32, 152), (16384, 32, 700, 64, 152),
    (4096, 128, 100, 64, 8), (0, 64, 6000, 8, 152), (2048, 40, 15, 24, 3)])
def test_plans_cover_their_trees(prefix, branches, tokens, h_q, sms):
    """Every (branch, page) once: pieces of two pages where the pass is small, longer ones elsewhere."""
    parent = [-1] * branches if prefix == 0 else [-1] + [0] * branches
    lens = [tokens + i % 3 for i in range(branches)]
    first = 0 if prefix == 0 else 1
    tree = W.build_tree("cover", parent, ([prefix] if prefix else []) + lens, list(range(first, first + branches)),
                        num_q_heads=h_q, num_kv_heads=8, head_dim=128, mode="fp4", values=False)
    with Plan.for_tree(tree, host_only=True, num_sms=sms) as plan:
        verify_plan(tree, plan)


def test_workloads_of_the_shape():
    with pytest.raises(ValueError):
        W.figure3_tree(d=128, mode="fp4")
    tree = W.figure3_tree(d=128, mode="fp4", values=False)
    assert tree.kv_elem_bytes() * 128 == 72
