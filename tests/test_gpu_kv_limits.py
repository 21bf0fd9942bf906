"""The cache's limits: the most key/value heads, a call that is more rows than one
launch numbers, and caches that are refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def cache(layers, pages, heads, page, dim):
    byte = dict(dtype=torch.uint8, device="cuda")
    return (torch.zeros((layers, pages, heads, page, dim), **byte), torch.zeros((layers, pages, heads, page, dim), **byte),
            torch.zeros((layers, pages, heads, page), **byte), torch.zeros((layers, pages, heads, page), **byte))


def test_many_heads_in_one_call(salt_lib, ctx):
    """1024 heads: a launch takes some thousand tokens, so one call is several launches; the bytes
    are those of calls of a few tokens, and they read back alike."""
    heads, dim, page, tokens = 1024, 64, 16, 2100
    pages = -(-tokens // page)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((tokens, heads, dim), generator=g, device="cuda").bfloat16() for _ in range(2))
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens].int()
    whole, parts = cache(1, pages, heads, page, dim), cache(1, pages, heads, page, dim)
    one, other = salt_lib.salt_kv_create(ctx, *whole), salt_lib.salt_kv_create(ctx, *parts)
    salt_lib.salt_kv_write(one, 0, k, v, slots)
    for t in range(0, tokens, 300):
        salt_lib.salt_kv_write(other, 0, k[t:t + 300], v[t:t + 300], slots[t:t + 300])
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)
    rk, rv = torch.empty_like(k), torch.empty_like(v)
    salt_lib.salt_kv_read(one, 0, slots, rk, rv)
    for t in range(0, tokens, 700):
        sk, sv = torch.empty_like(k[t:t + 700]), torch.empty_like(v[t:t + 700])
        salt_lib.salt_kv_read(other, 0, slots[t:t + 700], sk, sv)
        assert torch.equal(sk, rk[t:t + 700]) and torch.equal(sv, rv[t:t + 700])
    # half a code's step: a row's largest is at least 224 codes, steps are 32 there and fall with the value
    top = k.float().abs().amax(-1, keepdim=True)
    assert ((rk.float() - k.float()).abs() <= torch.maximum(k.float().abs() * 2.0 ** -4, top * 2.0 ** -17)).all()
    assert salt_lib.salt_get_device_error(ctx) == 0


@pytest.mark.parametrize("shape", [(1, 2, 1025, 16, 64), (1, 2, 1, 24, 64), (1, 2, 1, 256, 64), (1, 2, 1, 16, 96), (1, 2, 1, 16, 256)])
def test_caches_that_are_refused(salt_lib, ctx, shape):
    with pytest.raises(salt_lib.SaltError):
        salt_lib.salt_kv_create(ctx, *cache(*shape))
