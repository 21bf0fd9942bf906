"""Units whose rows are split, call after call with other log-sums, none of them waited for: a part that was read before it was written would be the call's before."""
import pytest
import torch

from test_gpu_weights import Weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


@pytest.mark.parametrize("dim,heads,kv_heads,n", [(64, 4, 1, 900), (128, 8, 2, 500), (128, 1, 1, 1500)])
def test_parts_of_calls_that_follow_each_other(salt_lib, ctx, dim, heads, kv_heads, n):
    w = Weights(salt_lib, ctx, [n], [n], heads=heads, kv_heads=kv_heads, dim=dim, page=64, seed=n)
    w.build()
    sums = [(w.lse + 0.5 * i).cuda() for i in range(4)]
    first = [w.check(lse=x) for x in sums]
    q = w.q.cuda()
    got = [w.w.cuda() for _ in range(60)]
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        salt_lib.salt_attn_weights(w.plan, 0, q, sums[i % 4], w.scale, x, 1.0)
    torch.cuda.synchronize()
    assert all(torch.equal(x.cpu(), first[i % 4]) for i, x in enumerate(got))
    assert salt_lib.salt_get_device_error(ctx) == 0
