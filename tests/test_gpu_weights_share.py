"""Lists of few rows beside lists of many: sharing the SMs costs no more than one kind after the other would."""
import pytest
import torch

from test_gpu_weights_replays import timed

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads,requests,own,groups,prompt", [(32, 8, 200, 1750, 3, 2000), (64, 8, 256, 1000, 2, 1000), (4, 1, 256, 1000, 8, 8192),
                                                                       (32, 8, 64, 500, 4, 4096)])
def test_both_kinds_of_lists(salt_lib, ctx, dim, heads, kv_heads, requests, own, groups, prompt):
    """Requests decoding behind prompts that many share.  (Fixed costs a second time make up for what the shares miss; with shares fitted to few requests both
    took 1.8 times as long as either after the other.)"""
    g = torch.Generator(device="cuda").manual_seed(dim)
    r = torch.Generator().manual_seed(requests)
    kv_len = torch.randint(own // 4, 2 * own - own // 4, (requests,), generator=r).tolist()
    group = torch.randint(0, groups, (requests,), generator=r).tolist()
    ptr = [0]
    for n in kv_len + [prompt] * groups:
        ptr.append(ptr[-1] + -(-n // PAGE))
    shape = (1, ptr[-1], kv_heads, PAGE)
    k = torch.randint(0, 0x70, shape + (dim,), dtype=torch.uint8, device="cuda", generator=g)
    e = torch.full(shape, 118, dtype=torch.uint8, device="cuda")
    plan = salt_lib.salt_attn_create(salt_lib.salt_kv_create(ctx, k, k, e, e), heads, requests, requests, ptr[-1], groups)
    salt_lib.salt_attn_track(plan)
    q = torch.randn((requests, heads, dim), device="cuda", generator=g).bfloat16()
    lse = torch.full((requests, heads), 20.0, device="cuda")
    w = torch.zeros(shape, device="cuda")
    own_ptr, own_pages = ptr[:requests + 1], list(range(ptr[requests]))
    pre_ptr, pre_pages = [n - ptr[requests] for n in ptr[requests:]], list(range(ptr[requests], ptr[-1]))

    def took(*batch):
        salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([1] * requests, *batch))
        return timed(lambda: salt_lib.salt_attn_weights(plan, 0, q, lse, 0.1, w, 1.0), 20)
    both = took(kv_len, own_ptr, own_pages, group, [prompt] * groups, pre_ptr, pre_pages)
    rows = took(kv_len, own_ptr, own_pages)
    chunks = took([0] * requests, [0] * (requests + 1), [], group, [prompt] * groups, pre_ptr, pre_pages)
    assert both <= 1.15 * (rows + chunks), f"{both:.1f} us for both, {rows:.1f} and {chunks:.1f} alone"
    assert salt_lib.salt_get_device_error(ctx) == 0
