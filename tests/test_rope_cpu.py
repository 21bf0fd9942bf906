"""What the rotation's calls refuse without a GPU, and its 64-bit definition
against other ways to write it."""
import ctypes
import math

import pytest
import torch

from rope_reference import angles, frequencies, rotate


def test_null_handles(salt_lib):
    lib, out = salt_lib._lib, ctypes.c_void_p(1)
    cfg = salt_lib._rope_config(64, 0, 0, None, 1.0, 1e-6, 0.0)
    assert lib.salt_rope_create(None, ctypes.byref(cfg), ctypes.byref(out)) == 1 and not out.value
    assert lib.salt_rope_create(None, ctypes.byref(cfg), None) == 1
    assert lib.salt_rope_apply(None, 1, *[None, 0, 1] * 2, None, None, None, None, 0, None, 0, None) == 1
    assert lib.salt_rope_write(None, None, 0, 1, None, 0, 1, None, 0, None, 0, None, None, None, None, None, 0, None) == 1
    lib.salt_rope_destroy(None)
    salt_lib.salt_rope_destroy(None)


def test_tensors_are_checked_before_the_call(salt_lib):
    rope = object.__new__(salt_lib.Rope)
    rope.ctx, rope.handle, rope.head_dim = None, None, 64
    x, i = torch.zeros((4, 2, 64), dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for args in ((x, x, i, x, x), (x[0], x, i, x, x)):   # host tensors, a matrix
        with pytest.raises(ValueError):
            salt_lib.salt_rope_apply(rope, *args)


def test_definition():
    """A rotation keeps lengths, turns by the difference of positions and is
    the product of complex numbers; far angles go by exact remainders."""
    x = torch.randn((5, 2, 64), dtype=torch.float64)
    f = frequencies(64)
    y, _ = rotate(x, [0, 1, 7, 1000, 123456], f)
    assert torch.equal(y[0], x[0])
    assert torch.allclose(y.norm(dim=-1), x.norm(dim=-1), rtol=1e-12)
    a, b = rotate(x[:1], [1007], f)[0], rotate(rotate(x[:1], [1000], f)[0], [7], f)[0]
    assert torch.allclose(a, b, rtol=0, atol=1e-12)
    z = torch.view_as_complex(x.unflatten(-1, (32, 2)))
    t = torch.tensor([3.0, 0.0, -2.0, 11.0, 5.0], dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    turned = torch.view_as_real(z * torch.polar(torch.ones_like(t), t)[:, None]).flatten(-2)
    assert torch.allclose(rotate(x, [3, 0, -2, 11, 5], f, interleaved=True)[0], turned, atol=1e-12)
    assert abs(float(angles([2 ** 31 - 1], [1.0])) - math.fmod(2 ** 31 - 1, 2 * math.pi)) < 1e-5
    n, _ = rotate(x, [0] * 5, [], norm=torch.ones(64), eps=1e-6)
    assert torch.allclose(n.square().mean(-1), torch.ones(5, 2, dtype=torch.float64), atol=1e-4)
