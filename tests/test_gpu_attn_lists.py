"""A batch's page lists are checked before any page number is read: pointers that go
down again would otherwise make the check read past the caller's array."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def plan(salt_lib):
    ctx = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    byte = dict(dtype=torch.uint8, device="cuda")
    shape = (1, 8, 2, 16, 64)
    cache = [torch.zeros(shape, **byte), torch.zeros(shape, **byte), torch.zeros(shape[:4], **byte), torch.zeros(shape[:4], **byte)]
    kv = salt_lib.salt_kv_create(ctx, *cache)
    p = salt_lib.salt_attn_create(kv, 4, 3, 4, 400, 3)
    yield p
    salt_lib.salt_attn_destroy(p)
    salt_lib.salt_kv_destroy(kv)
    salt_lib.salt_ctx_destroy(ctx)


def batch(salt, ptr, pages, lens, gptr=(0, 0), gpages=(), glens=(0,)):
    """The C structure itself, as the binding's own checks would not let all of these through.  Behind the
    last page that the lists have lie numbers that no cache has."""
    a = [np.ascontiguousarray(x, dtype=np.int32) for x in
         ([1] * len(lens), lens, ptr, list(pages) + [10 ** 9] * 300, [-1] * len(lens), glens, gptr, list(gpages) + [10 ** 9] * 300)]
    p = [x.ctypes.data for x in a]
    b = salt._attn_batch(len(lens), p[0], p[1], p[2], p[3], p[4], len(glens), p[5], p[6], p[7])
    b._keep, b._tokens = a, len(lens)
    return b


@pytest.mark.parametrize("bad", [
    dict(ptr=[0, 100, 5], pages=range(5), lens=[1600, 16]),                      # 100 pages' tokens, five pages
    dict(ptr=[0, 5, 200, 3], pages=range(3), lens=[16, 3000, 0]),
    dict(ptr=[0, 401, 5], pages=range(5), lens=[6400, 16]),                      # past max_pages
    dict(ptr=[0, 1], pages=[0], lens=[16], gptr=[0, 90, 2], gpages=[0, 1], glens=[1400, 16]),
])
def test_pointers_before_pages(salt_lib, plan, bad):
    with pytest.raises(salt_lib.SaltError) as e:
        salt_lib.salt_attn_build(plan, batch(salt_lib, **bad))
    assert e.value.name == "SALT_ERR_INVALID_ARG", str(e.value)


def test_good_lists_still_pass(salt_lib, plan):
    salt_lib.salt_attn_build(plan, batch(salt_lib, [0, 3, 3, 5], [7, 6, 5, 4, 3], [33, 0, 32], [0, 2], [1, 0], [17]))
    salt_lib.salt_attn_build(plan, batch(salt_lib, [0, 3, 5], [7, 6, 10 ** 9, 4, 3], [32, 32]))  # entries past a length's pages are not looked at
