"""Builds, weights and evictions that follow each other without a wait on the host: each call goes by the tables and numbers that were written just before it."""
import pytest
import torch

from test_gpu_evict import ARRAYS, Cache
from test_gpu_weights import Weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 4, 2), (128, 8, 8)])
def test_builds_and_weights(salt_lib, ctx, dim, heads, kv_heads):
    w = Weights(salt_lib, ctx, [1, 90, 3, 1], [70, 300, 5, 129], [0, -1, 0, 0], [200], heads=heads, kv_heads=kv_heads, dim=dim)
    b = w.batch
    batches = [dict(b, q_len=q, kv_len=kv, group=g) for q, kv, g in (
        (b["q_len"], b["kv_len"], b["group"]), ([1, 1, 1, 1], [70, 300, 5, 100], [-1] * 4), ([0, 95, 0, 0], [70, 95, 5, 129], [-1, 0, -1, -1]),
        ([90, 1, 3, 1], [90, 211, 3, 1], [0, 0, -1, -1]))]
    for x in batches:   # (pages for 90 tokens of the first request)
        x["kv_len"] = [min(n, 16 * (b["page_ptr"][i + 1] - b["page_ptr"][i])) for i, n in enumerate(x["kv_len"])]
    q, lse = w.q.cuda(), w.lse.clamp(min=0.0).cuda()

    def call(i, x):
        c = batches[i]
        salt_lib.salt_attn_build(w.plan, salt_lib.salt_attn_batch(c["q_len"], c["kv_len"], c["page_ptr"], c["pages"], c["group"], c["group_len"],
                                                                  c["group_page_ptr"], c["group_pages"]))
        salt_lib.salt_attn_weights(w.plan, 0, q, lse, w.scale, x, 0.5)
    want = []
    for i in range(len(batches)):
        want.append(w.w.cuda())
        call(i, want[-1])
        torch.cuda.synchronize()
    order = [0, 1, 2, 3, 1, 0, 3, 2, 0, 2, 1, 3] * 3
    got = [w.w.cuda() for _ in order]
    torch.cuda.synchronize()
    for i, x in zip(order, got):
        call(i, x)
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0
    assert all(torch.equal(x.view(torch.int32), want[i].view(torch.int32)) for i, x in zip(order, got))


@pytest.mark.parametrize("requests,kv_heads", [(2, 1), (40, 8)])
def test_numbers_written_just_before(salt_lib, ctx, requests, kv_heads):
    c = Cache(salt_lib, ctx, [300 + i for i in range(requests)], kv_heads=kv_heads, dim=64, page=16)
    scores = torch.randn(c.t["weights"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    fresh = [c.t[n].clone() for n in ARRAYS]
    keeps = [torch.full((requests,), k, dtype=torch.int32, device="cuda") for k in (40, 290, 0, 129, 400)]
    keep = torch.zeros((requests,), dtype=torch.int32, device="cuda")

    def results(together):
        out = []
        for k in keeps * 3:
            for n, x in zip(ARRAYS, fresh):
                c.t[n].copy_(x)
            kept = torch.full((2, requests, kv_heads, 400), -7, dtype=torch.int32, device="cuda")
            keep.copy_(k)
            salt_lib.salt_attn_evict(c.plan, 0, 2, keep, scores, kept, 1, 9, c.t["weights"])
            out.append([kept] + [c.t[n].clone() for n in ARRAYS])
            if not together:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return out
    for a, b in zip(results(False), results(True)):
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))
    assert salt_lib.salt_get_device_error(ctx) == 0
