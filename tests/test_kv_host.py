"""Refusals of the cache operators, through the C ABI, where no GPU is needed:
every call here is refused before anything would be launched."""
import ctypes

import numpy as np
import pytest

from paper_2608_24658_gb300 import _lib, build

A = 1 << 20          # an address that nothing reads: aligned, never dereferenced


@pytest.fixture(scope="module")
def lib():
    build.build()
    return _lib.load()


def _cfg(mode="bf16", **kw):
    f = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, mode=_lib.MODES.get(mode, mode),
             sm_scale=0.0)
    f.update(kw)
    return _lib.AttnConfig(**f)


def _rows(data=A, ts=1024, hs=128):
    return _lib.Rows(data, ts, hs)


def _rot(**kw):
    f = dict(rotary_dim=128, pairs=0, num_axes=1, freq_axis=None, turns=A, positions=A, position_stride=0)
    f.update(kw)
    return _lib.RotaryDesc(**f)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _write(lib, cfg=None, n=4, q=None, k=_rows(), v=_rows(), rot=None, slots=A, ks=None, vs=None,
           q_out=None, kp=A, vp=A, pages=10):
    return lib.parason_kv_write(_ref(cfg or _cfg()), n, _ref(q), _ref(k), _ref(v), _ref(rot), slots,
                                ks, vs, q_out, kp, vp, pages, None)


def _read(lib, cfg=None, n=4, slots=A, kp=A, vp=A, pages=10, ks=None, vs=None, k=_rows(), v=_rows()):
    return lib.parason_kv_read(_ref(cfg or _cfg()), n, slots, kp, vp, pages, ks, vs, _ref(k), _ref(v),
                               None)


def _scales(lib, cfg=None, n=4, k=_rows(), v=_rows(), rot=None, slots=None, acc=0, ks=A, vs=A):
    return lib.parason_kv_scales(_ref(cfg or _cfg("fp8")), n, _ref(k), _ref(v), _ref(rot), slots, acc,
                                 ks, vs, None)


BAD_CFG = [dict(num_kv_heads=3), dict(head_dim=96), dict(page_size=32), dict(mode=5), dict(num_q_heads=0)]


@pytest.mark.parametrize("bad", BAD_CFG)
def test_bad_configs(lib, bad):
    assert _write(lib, _cfg(**bad)) == _lib.EINVAL
    assert _read(lib, _cfg(**bad)) == _lib.EINVAL
    if "mode" not in bad:
        assert _scales(lib, _cfg("fp8", **bad)) == _lib.EINVAL


def test_shapes_without_a_kernel(lib):
    assert _write(lib, _cfg("fp8", head_dim=64), ks=A, vs=A) == _lib.EUNSUPPORTED
    assert _read(lib, _cfg("fp8", head_dim=64), ks=A, vs=A) == _lib.EUNSUPPORTED
    most = (2 ** 31 - 1) // 32
    assert _write(lib, pages=most + 1) == _lib.EUNSUPPORTED
    assert _read(lib, pages=most + 1) == _lib.EUNSUPPORTED
    assert _scales(lib, _cfg("bf16")) == _lib.EINVAL
    many = dict(num_q_heads=16386, num_kv_heads=2)
    assert _write(lib, _cfg(**many)) == _lib.EUNSUPPORTED
    assert _read(lib, _cfg(num_q_heads=16385, num_kv_heads=16385), pages=1) == _lib.EUNSUPPORTED
    assert _scales(lib, _cfg("fp8", num_q_heads=16385, num_kv_heads=16385)) == _lib.EUNSUPPORTED


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n=2 ** 31), dict(pages=-1), dict(k=None), dict(v=None), dict(slots=None),
    dict(slots=A + 2), dict(kp=None), dict(vp=None), dict(kp=A + 8), dict(vp=A + 4),
    dict(k=_rows(None)), dict(k=_rows(A + 2)), dict(v=_rows(ts=1028)), dict(v=_rows(hs=100)),
    dict(k=_rows(ts=-1024)), dict(q=_rows()), dict(q=_rows(), q_out=A + 2), dict(q=_rows(A + 8), q_out=A),
    # in place, but not as q_out lies
    dict(q=_rows(ts=1032), q_out=A), dict(q=_rows(ts=128, hs=512), q_out=A)])
def test_write_refusals(lib, bad):
    assert _write(lib, **bad) == _lib.EINVAL


@pytest.mark.parametrize("bad", [dict(ks=None), dict(vs=None), dict(ks=A + 1)])
def test_e4m3_needs_scales(lib, bad):
    assert _write(lib, _cfg("fp8"), **dict(dict(ks=A, vs=A), **bad)) == _lib.EINVAL
    assert _read(lib, _cfg("fp8"), **dict(dict(ks=A, vs=A), **bad)) == _lib.EINVAL


@pytest.mark.parametrize("bad", [
    dict(rotary_dim=0), dict(rotary_dim=136), dict(rotary_dim=24), dict(rotary_dim=-16), dict(pairs=2),
    dict(pairs=-1), dict(num_axes=0), dict(num_axes=5), dict(turns=None), dict(positions=None),
    dict(turns=A + 4), dict(positions=A + 1), dict(num_axes=2, position_stride=-4)])
def test_rotary_refusals(lib, bad):
    assert _write(lib, rot=_rot(**bad)) == _lib.EINVAL
    if "rotary_dim" in bad or "pairs" in bad:
        assert _scales(lib, rot=_rot(**bad)) == _lib.EINVAL


def test_axis_past_the_axes(lib):
    table = np.zeros(64, np.uint8)
    table[63] = 2
    rot = _rot(num_axes=2, position_stride=4, freq_axis=table.ctypes.data)
    assert _write(lib, rot=rot) == _lib.EINVAL
    # the rotary part is checked for an empty batch too, which launches nothing
    assert _write(lib, n=0, rot=rot) == _lib.EINVAL
    assert _write(lib, n=0, k=None, v=None, slots=None, kp=None, vp=None) == _lib.OK
    assert _write(lib, n=0, k=None, v=None, slots=None, kp=None, vp=None, rot=_rot(positions=None)) == _lib.OK


def test_more_rows_than_a_grid(lib):
    n = 2 ** 31 - 1
    big = [_rows(ts=4096, hs=128) for _ in range(2)]
    for mode, call in (("bf16", _read), ("fp8", _scales)):
        cfg = _cfg(mode, num_q_heads=16, num_kv_heads=16)
        assert call(lib, cfg, n=n, k=big[0], v=big[1]) == _lib.EUNSUPPORTED


@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(slots=None), dict(kp=None), dict(vp=A + 8), dict(k=None), dict(v=_rows(A + 4)),
    dict(k=_rows(ts=64)), dict(v=_rows(hs=64)), dict(k=_rows(ts=0)), dict(k=_rows(hs=0)),
    # rows that reach into the next token's, or the next head's (heads first)
    dict(k=_rows(ts=128, hs=128)), dict(v=_rows(ts=248, hs=128)), dict(k=_rows(ts=136, hs=528)),
    dict(v=_rows(ts=1024, hs=1024))])
def test_read_refusals(lib, bad):
    assert _read(lib, **bad) == _lib.EINVAL
    assert _read(lib, n=0, slots=None, kp=None, vp=None, k=None, v=None) == _lib.OK


@pytest.mark.parametrize("bad", [dict(n=-1), dict(k=None), dict(v=None), dict(acc=2), dict(ks=None),
                                 dict(vs=None), dict(ks=A + 2), dict(slots=A + 1), dict(k=_rows(A + 2)),
                                 dict(v=_rows(hs=4))])
def test_scales_refusals(lib, bad):
    assert _scales(lib, **bad) == _lib.EINVAL
    # raising scales by no tokens launches nothing
    assert _scales(lib, n=0, k=None, v=None, acc=1) == _lib.OK


def test_null_config(lib):
    assert lib.parason_kv_write(None, 0, None, None, None, None, None, None, None, None, None, None, 0,
                                None) == _lib.EINVAL
    assert lib.parason_kv_read(None, 0, None, None, None, 0, None, None, None, None, None) == _lib.EINVAL
    assert lib.parason_kv_scales(None, 0, None, None, None, None, 0, None, None, None) == _lib.EINVAL


def test_turns_of_frequencies(lib):
    """inv_freq / (2 pi) modulo 1 in 2^-64, against exact integers; and the angles they give."""
    def pi_times_2_to(bits):
        def arctan_inverse(x):
            one = term = (1 << (bits + 64)) // x
            n, sign = 3, -1
            while term:
                term //= x * x
                one += sign * (term // n)
                n, sign = n + 2, -sign
            return one
        return (4 * (4 * arctan_inverse(5) - arctan_inverse(239))) >> 64

    rng = np.random.default_rng(0)
    f = np.concatenate([(1e4 ** (-np.arange(64) / 64)), [0.0, -0.5, 1e-45, 1e-38, 2.0 ** 40, -2.0 ** 64, 123456.789],
                        rng.standard_normal(50) * 10.0 ** rng.integers(-20, 15, 50)]).astype(np.float32)
    turns = np.empty(len(f), np.uint64)
    assert lib.parason_rotary_turns(f.ctypes.data, len(f), turns.ctypes.data) == _lib.OK
    pi = pi_times_2_to(600)
    for x, got in zip(f, turns):
        m, e = np.frexp(np.float64(x))
        n = int(m * 2 ** 53)                     # x = n 2^(e - 53)
        shift = int(e) - 53 + 64 + 600           # x / 2 pi in 2^-64 = n 2^(e - 53 + 64) 2^600 / (2 pi 2^600)
        want = ((n << shift if shift >= 0 else 0) + pi) // (2 * pi) if shift >= 0 else 0
        assert (int(got) - want) % 2 ** 64 in (0, 1, 2 ** 64 - 1), (x, got, want % 2 ** 64)
    for bad in (np.inf, -np.inf, np.nan, 2.0 ** 65):
        one = np.array([0.5, bad], np.float32)
        assert lib.parason_rotary_turns(one.ctypes.data, 2, turns.ctypes.data) == _lib.EINVAL
    assert lib.parason_rotary_turns(None, 1, turns.ctypes.data) == _lib.EINVAL
    assert lib.parason_rotary_turns(f.ctypes.data, 1, None) == _lib.EINVAL
    assert lib.parason_rotary_turns(f.ctypes.data, -1, turns.ctypes.data) == _lib.EINVAL
    assert lib.parason_rotary_turns(None, 0, None) == _lib.OK
