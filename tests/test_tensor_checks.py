"""The binding's one-call looks at tensors: they answer for what is plainly right, and leave
everything else to the binding's own checks."""
import struct

import numpy as np
import pytest
import torch

from paper_2608_24658_gb300 import _lib, build
from paper_2608_24658_gb300.api import kv_read, kv_slots, kv_write


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    _lib.load()


class Sub(torch.Tensor):
    pass


def test_nothing_on_the_cpu():
    x = torch.zeros((2, 3), dtype=torch.int32)
    for call in (lambda: _lib.flat(x, torch.int32, 0, 2, 3), lambda: _lib.flat(x, torch.int32, -1, 2, 3),
                 lambda: _lib.flat(None, torch.int32, 0), lambda: _lib.flat(np.zeros(3), torch.int32, 0, 3),
                 lambda: _lib.flat(), lambda: _lib.flat(x), lambda: _lib.rows(x, torch.int32, 0, 1, 2, 3),
                 lambda: _lib.rows(), lambda: _lib.alike(x, x), lambda: _lib.alike(x), lambda: _lib.alike(None, x),
                 lambda: _lib.flat(torch.zeros((2, 3), device="meta"), torch.float32, 0, 2, 3)):
        assert call() is None


@pytest.mark.gpu
def test_flat():
    x = torch.zeros((4, 6), dtype=torch.int32, device="cuda")
    assert _lib.flat(x, torch.int32, 0, 4, 6) == x.data_ptr()
    assert _lib.flat(x[1:], torch.int32, 0, 3, 6) == x.data_ptr() + 24
    assert _lib.flat(torch.nn.Parameter(x.float()), torch.float32, 0, 4, 6)
    assert _lib.flat(x[:0], torch.int32, 0, 0, 6) is not None
    for t, dtype, dev, size in ((x, torch.float32, 0, (4, 6)), (x, torch.int32, 1, (4, 6)), (x, torch.int32, 0, (4, 7)),
                                (x, torch.int32, 0, (24,)), (x.t(), torch.int32, 0, (6, 4)), (x[:, :3], torch.int32, 0, (4, 3)),
                                (x, torch.int32, 0, (4, 6.0)), (x, torch.int32, 0, (4, 2 ** 70)), (x, torch.int32, 2 ** 70, (4, 6)),
                                (x, "int32", 0, (4, 6)), (x.as_subclass(Sub), torch.int32, 0, (4, 6))):
        assert _lib.flat(t, dtype, dev, *size) is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows(dtype):
    x = torch.zeros((5, 48, 64), dtype=dtype, device="cuda")
    part = x[:, 8:40]
    assert _lib.rows(part, dtype, 0, 5, 32, 64) == struct.pack("@Pqq", part.data_ptr(), 48 * 64, 64)
    assert _lib.rows(x.transpose(0, 1), dtype, 0, 48, 5, 64) == struct.pack("@Pqq", x.data_ptr(), 64, 48 * 64)
    odd = torch.zeros(5 * 48 * 64 + 1, dtype=dtype, device="cuda")[1:].view(5, 48, 64)
    for t, size in ((x[..., ::2], (5, 48, 32)), (odd, (5, 48, 64)), (x[..., 1:33], (5, 48, 32)), (x, (5, 48, 65)),
                    (x.view(5, 48, 1, 64), (5, 48, 64)), (x.flatten().as_strided((5, 4, 32), (66 * 4 + 2, 64, 1)), (5, 4, 32))):
        assert _lib.rows(t, dtype, 0, *size) is None


@pytest.mark.gpu
def test_alike():
    a, b = (torch.zeros((3, 2, 72), dtype=torch.uint8, device="cuda") for _ in range(2))
    assert _lib.alike(a, b) == (torch.uint8, 0, a.data_ptr(), b.data_ptr(), (3, 2, 72))
    for c in (b.view(torch.int8), b[:2], b.transpose(0, 1), b.cpu(), b.as_subclass(Sub), None):
        assert _lib.alike(a, c) is None
        assert _lib.alike(c, a) is None


@pytest.mark.gpu
def test_the_same_without_them(monkeypatch):
    """The binding's own checks take the same calls, with the same results."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v, q = (torch.randn((20, h, 128), generator=gen, device="cuda").to(torch.bfloat16) for h in (2, 2, 8))
    i = dict(dtype=torch.int32, device="cuda")

    def run():
        pools = [torch.zeros((4, 2, 1152), dtype=torch.uint8, device="cuda") for _ in range(2)]
        ones = torch.full((2,), 0.5, device="cuda")
        table = torch.full((2, 2), -1, **i)
        slots, positions = kv_slots(table, torch.zeros(2, **i), torch.tensor([3, 17], **i), 20,
                                    free_pages=torch.tensor([3, 1, 0], **i))
        q_out = kv_write(k, v, *pools, slots, q=q, q_out=torch.empty_like(q), k_scale=ones, v_scale=ones)
        return [slots, positions, table, q_out, *pools, *kv_read(*pools, slots, k_scale=ones, v_scale=ones)]

    fast = run()
    for name in ("flat", "rows", "alike"):
        monkeypatch.setattr(_lib, name, _lib._unknown)
    assert all(torch.equal(x, y) for x, y in zip(fast, run()))
