"""Lists of pages that no token needs, given without an array, are refused: the build
copies the lists whole."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups", [False, True])
def test_lists_without_an_array(salt_lib, groups):
    ctx = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    byte = dict(dtype=torch.uint8, device="cuda")
    shape = (1, 8, 2, 16, 64)
    cache = [torch.zeros(shape, **byte), torch.zeros(shape, **byte), torch.zeros(shape[:4], **byte), torch.zeros(shape[:4], **byte)]
    kv = salt_lib.salt_kv_create(ctx, *cache)
    plan = salt_lib.salt_attn_create(kv, 4, 1, 1, 4, 1)
    zero, one, lists = (np.array(x, np.int32) for x in ([0], [1], [0, 2]))
    none, group = np.array([0, 0], np.int32), np.array([-1], np.int32)
    p = lambda a: a.ctypes.data  # noqa: E731
    b = salt_lib._attn_batch(1, p(one), p(zero), p(none if groups else lists), None, p(group), int(groups), p(zero), p(lists), None)
    b._tokens = 1
    with pytest.raises(salt_lib.SaltError) as e:
        salt_lib.salt_attn_build(plan, b)
    assert e.value.name == "SALT_ERR_INVALID_ARG"
    salt_lib.salt_attn_destroy(plan)
    salt_lib.salt_kv_destroy(kv)
    salt_lib.salt_ctx_destroy(ctx)
