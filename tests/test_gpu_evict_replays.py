"""A captured eviction replayed on longer lines: its rows are moved by as many CTAs as a direct call's."""
import numpy as np
import pytest
import torch

from keeping_reference import evict
from test_gpu_evict import ARRAYS, Cache
from test_gpu_weights_replays import timed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def test_ctas_of_the_move(salt_lib, ctx):
    """A line of 4,000 tokens cut to 3,500, captured when it had 10: by the one CTA that 10 tokens need it took 63 us where CTAs of its own number take 15."""
    c = Cache(salt_lib, ctx, [4000], kv_heads=1, dim=128, page=64, layers=1)
    scores = torch.randn(c.t["weights"].shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    keep = torch.tensor([3500], dtype=torch.int32, device="cuda")
    kept = torch.full((1, 1, 1, 3500), -7, dtype=torch.int32, device="cuda")

    def call():
        salt_lib.salt_attn_evict(c.plan, 0, 1, keep, scores, kept, 0, 100, c.t["weights"])
    before = c.host()
    c.build(kv_len=[10])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            call()
    c.build()
    torch.cuda.synchronize()
    arrays, want = evict(before, c.batch, 64, [0], [3500], scores.cpu().numpy(), np.full((1, 1, 1, 3500), -7), 0, 100)
    call()
    torch.cuda.synchronize()
    assert np.array_equal(kept.cpu().numpy(), want)
    assert all(np.array_equal(a.view(np.uint8), b.view(np.uint8)) for a, b in zip(c.host(), arrays))
    direct = torch.cuda.CUDAGraph()
    with torch.cuda.graph(direct):
        for _ in range(10):
            call()
    took, best = timed(graph.replay, 5) / 10, timed(direct.replay, 5) / 10
    assert took < 1.5 * best, f"{took:.1f} us as captured for few tokens, {best:.1f} us as captured for these"
    assert np.array_equal(kept.cpu().numpy(), want) and salt_lib.salt_get_device_error(ctx) == 0
