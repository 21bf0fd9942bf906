"""Evictions whose chunks of rows all write over what others read: every row moves by little, again and again, bit for bit."""
import numpy as np
import pytest
import torch

from keeping_reference import evict
from test_gpu_evict import ARRAYS, Cache, scores_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


@pytest.mark.parametrize("dim,page,lens,kv_heads,layers", [(64, 16, [4097, 3001], 8, 2), (128, 64, [20001], 4, 1), (128, 16, [700] * 24, 4, 3)])
@pytest.mark.parametrize("by", [1, 63, 65, 129])
def test_every_chunk_waits(salt_lib, ctx, dim, page, lens, kv_heads, layers, by):
    """The last tokens are kept, so that a row moves `by` places and each chunk's place is where one or two others still lie."""
    c = Cache(salt_lib, ctx, lens, kv_heads=kv_heads, dim=dim, page=page, layers=layers, seed=by)
    scores = torch.zeros_like(c.t["weights"])
    left = [x.reshape(x.shape[:4] + (-1,)).view(np.uint8) for x in c.host()]
    for _ in range(5):
        keep = [n - by for n in lens]
        kept = torch.full((layers, len(lens), kv_heads, max(keep)), -7, dtype=torch.int32, device="cuda")
        salt_lib.salt_attn_evict(c.plan, 0, layers, torch.tensor(keep, dtype=torch.int32, device="cuda"), scores, kept, 0, 1 << 30, c.t["weights"])
        torch.cuda.synchronize()
        assert salt_lib.salt_get_device_error(ctx) == 0
        for b, n in enumerate(lens):
            pages = np.array(c.batch["pages"][c.batch["page_ptr"][b]:c.batch["page_ptr"][b + 1]])
            j = np.arange(n)
            P, O = pages[j // page], j % page
            for x in left:
                x[:, P[:n - by], :, O[:n - by]] = x[:, P[by:], :, O[by:]]
            assert bool((kept[:, b, :, :n - by] == torch.arange(by, n, device="cuda")).all())
        for name, a, b in zip(ARRAYS, c.host(), left):
            assert np.array_equal(a.reshape(a.shape[:4] + (-1,)).view(np.uint8), b), name
        lens = keep
        c.build(kv_len=lens)


@pytest.mark.parametrize("dim,page", [(128, 32), (64, 16)])
@pytest.mark.parametrize("requests,part", [(40, 1.0), (40, 0.6), (20, 0.9), (31, 0.02)])
def test_whole_lines_and_shared_ones(salt_lib, ctx, dim, page, requests, part):
    """Lines of many chunks, more and fewer than a round of them a CTA, among requests that lose nothing."""
    r = np.random.RandomState(requests)
    lens = [int(n) for n in r.randint(300, 1800, requests)]
    keep = [int(n * r.uniform(0.3, 0.99)) if r.rand() < part else n for n in lens]
    keep[-1] = lens[-1] - 1
    c = Cache(salt_lib, ctx, lens, kv_heads=4, dim=dim, page=page, layers=4, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    c.check(keep, torch.randn(c.t["weights"].shape, device="cuda", generator=g), 4, 100)


@pytest.mark.parametrize("kind", ["ties", "close", "strange"])
def test_more_lines_than_a_wave(salt_lib, ctx, kind):
    """Lines up to the longest that the smallest CTAs search."""
    r = np.random.RandomState(7)
    lens = [2048, 1, 2047] + [int(n) for n in r.randint(1, 900, 157)]
    c = Cache(salt_lib, ctx, lens, kv_heads=8, dim=64, page=64, layers=1, seed=8)
    c.check([int(n * r.uniform(0.0, 1.0)) for n in lens], scores_of(c, kind), 2, 5)


def test_captured_for_whole_lines(salt_lib, ctx):
    """A captured call of many lines, replayed where fewer requests, none, or too many are there, and where none loses a token."""
    r = np.random.RandomState(11)
    lens = [int(n) for n in r.randint(200, 900, 30)]
    c = Cache(salt_lib, ctx, lens, kv_heads=4, dim=128, page=32, layers=3, seed=12)
    scores, keep = scores_of(c, "ties"), [int(n * r.uniform(0.2, 1.1)) for n in lens]
    keep_d, places = torch.zeros(30, dtype=torch.int32, device="cuda"), 1000
    fresh, kept = [c.t[n].clone() for n in ARRAYS], torch.empty((3, 30, 4, places), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        salt_lib.salt_attn_evict(c.plan, 0, 3, keep_d, scores, kept, 3, 20, c.t["weights"])
    for n, left in ((30, keep), (30, lens), (7, keep), (0, keep), (30, [0] * 30), (30, keep[::-1])):
        for name, x in zip(ARRAYS, fresh):
            c.t[name].copy_(x)
        kept.fill_(-7)
        left = left[:n]
        keep_d[:n] = torch.tensor(left, dtype=torch.int32, device="cuda")
        b = dict(c.batch, kv_len=lens[:n], page_ptr=c.batch["page_ptr"][:n + 1])
        c.build(**b)
        graph.replay()
        torch.cuda.synchronize()
        arrays, want = evict([x.cpu().numpy() for x in fresh], b, 32, range(3), left, scores.cpu().numpy(), np.full((3, n, 4, places), -7), 3, 20)
        assert np.array_equal(kept.cpu().numpy()[:, :n], want) and bool((kept[:, n:] == -7).all())
        assert all(np.array_equal(c.t[name].cpu().numpy().view(np.uint8), a.view(np.uint8)) for name, a in zip(ARRAYS, arrays))
        assert salt_lib.salt_get_device_error(ctx) == 0
    # more requests than at the capture
    c.build(**dict(c.batch, kv_len=lens[:28], page_ptr=c.batch["page_ptr"][:29]))
    small, kept = torch.cuda.CUDAGraph(), torch.empty((3, 28, 4, places), dtype=torch.int32, device="cuda")
    with torch.cuda.graph(small):
        salt_lib.salt_attn_evict(c.plan, 0, 3, keep_d[:28], scores, kept, 3, 20, c.t["weights"])
    c.build()
    before = c.host()
    small.replay()
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0x80
    assert all(np.array_equal(a.view(np.uint8), b.view(np.uint8)) for a, b in zip(before, c.host()))
