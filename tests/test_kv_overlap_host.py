"""Calls whose outputs would share memory are refused before a launch (no GPU needed)."""
import pytest

from paper_2608_24658_gb300 import _lib
from tests.test_kv_host import A, _cfg, _read, _rows, _write, lib  # noqa: F401

B, C, D, E = A + (1 << 16), A + (1 << 17), A + (1 << 18), A + (1 << 19)


@pytest.mark.parametrize("mode", ["bf16", "fp32", "fp8"])
def test_outputs_in_one_place(lib, mode):  # noqa: F811
    scales = dict(ks=A, vs=A)
    # K and V of a read, of a pool, rotated queries over keys or values
    assert _read(lib, _cfg(mode), k=_rows(B), v=_rows(B), **scales) == _lib.EINVAL
    assert _write(lib, _cfg(mode), k=_rows(B), v=_rows(C), kp=D, vp=D, **scales) == _lib.EINVAL
    for q_out in (B, C):
        assert _write(lib, _cfg(mode), q=_rows(A), k=_rows(B), v=_rows(C), kp=D, vp=E, q_out=q_out,
                      **scales) == _lib.EINVAL
    # nothing is written: nothing is in the way
    assert _read(lib, _cfg(mode), n=0, k=_rows(B), v=_rows(B), **scales) == _lib.OK
    assert _write(lib, _cfg(mode), n=0, k=_rows(B), v=_rows(C), kp=D, vp=D, **scales) == _lib.OK
