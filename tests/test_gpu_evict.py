"""Eviction from the cache, bit for bit against the definition: which tokens are kept, where
they go, what stays as it was; ties, NaN, long lines, streams, graphs and
refusals; and the operators of a cache whose tokens come and go together."""
import math

import numpy as np
import pytest
import torch

from attn_reference import attention, value
from keeping_reference import add_weights, check_weights, evict
from rope_reference import check_bf16, frequencies, rotate
from test_gpu_attn import compare

pytestmark = pytest.mark.gpu

ARRAYS = ("k", "v", "k_exp", "v_exp", "weights")


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


class Cache:
    """A cache of random bytes and a built plan of requests in it."""

    def __init__(self, salt, ctx, kv_len, kv_heads=2, dim=64, page=16, layers=2, seed=0, spare=1, q_len=None):
        self.salt, self.ctx, self.kv_len, self.page, self.layers, self.kv_heads = salt, ctx, kv_len, page, layers, kv_heads
        need = [-(-n // page) + (spare if i % 2 else 0) for i, n in enumerate(kv_len)]   # some lists longer than they need be
        r = np.random.RandomState(seed)
        n_pages = sum(need) + 2
        order = r.permutation(n_pages).tolist()
        ptr = np.cumsum([0] + need).tolist()
        self.batch = dict(kv_len=kv_len, page_ptr=ptr, pages=order[:ptr[-1]])
        shape = (layers, n_pages, kv_heads, page)
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda s: torch.randint(0, 256, s, dtype=torch.uint8, device="cuda", generator=g)  # noqa: E731
        self.t = dict(k=rand(shape + (dim,)), v=rand(shape + (dim,)), k_exp=rand(shape), v_exp=rand(shape),
                      weights=torch.randn(shape, device="cuda", generator=g))
        self.kv = salt.salt_kv_create(ctx, *(self.t[n] for n in ARRAYS[:4]))
        self.plan = salt.salt_attn_create(self.kv, kv_heads, max(1, len(kv_len)), max(1, len(kv_len)), max(1, ptr[-1]))
        salt.salt_attn_track(self.plan)
        self.build()

    def build(self, **kw):
        b = {**self.batch, **kw}
        self.salt.salt_attn_build(self.plan, self.salt.salt_attn_batch([0] * len(b["kv_len"]), b["kv_len"], b["page_ptr"], b["pages"]))

    def host(self):
        return [self.t[n].cpu().numpy() for n in ARRAYS]

    def check(self, keep, scores, first=0, recent=0, layer=0, n_layers=None, places=None, weights=True, flags=0, stream=None):
        n_layers = self.layers - layer if n_layers is None else n_layers
        places = max([0] + keep) if places is None else places
        kept = torch.full((n_layers, len(keep), self.kv_heads, places), -7, dtype=torch.int32, device="cuda")
        before = self.host()
        n = 5 if weights else 4
        arrays, want = evict(before[:n], self.batch, self.page, range(layer, layer + n_layers), keep, scores.cpu().numpy(), kept.cpu().numpy(), first,
                             recent)
        keep_d = torch.tensor(keep, dtype=torch.int32, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.salt.salt_attn_evict(self.plan, layer, n_layers, keep_d, scores, kept, first, recent, self.t["weights"] if weights else None, stream)
        torch.cuda.synchronize()
        assert self.salt.salt_get_device_error(self.ctx) == flags
        assert np.array_equal(kept.cpu().numpy(), want)
        for name, a, b in zip(ARRAYS, self.host(), arrays + before[n:]):
            assert np.array_equal(a.view(np.uint8), b.view(np.uint8)), name


def scores_of(c, kind, seed=5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = torch.randn(c.t["weights"].shape, device="cuda", generator=g)
    if kind == "ties":
        s = torch.randint(-2, 3, s.shape, device="cuda", generator=g).float() * 0.5
        s[s == 0] *= torch.where(torch.rand(s[s == 0].shape, device="cuda", generator=g) < 0.5, -1.0, 1.0)   # both zeros
    elif kind == "equal":
        s.fill_(-3.25)
    elif kind == "close":    # that differ in their last digits
        s = (s.abs() * 8).round().int().add_(0x3F800000).view(torch.float32)
    elif kind == "strange":
        r = torch.rand(s.shape, device="cuda", generator=g)
        for lo, x in ((0.0, math.nan), (0.1, math.inf), (0.2, -math.inf), (0.3, 1e-45), (0.4, -1e-45), (0.5, 3.4e38), (0.6, -math.nan)):
            s[(r >= lo) & (r < lo + 0.1)] = x
    return s


@pytest.mark.parametrize("dim,page", [(64, 16), (64, 128), (128, 32), (128, 64)])
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "close", "strange"])
def test_ragged_requests(salt_lib, ctx, dim, page, kind):
    lens = [1, 40, 0, 17, 300, 128, 1025, 64]
    c = Cache(salt_lib, ctx, lens, dim=dim, page=page, seed=dim + page)
    c.check([1, 20, 0, 16, 77, 128, 600, 1], scores_of(c, kind))
    c.check([0, 39, 5, 1, 299, 3, 1024, 63], scores_of(c, kind, 6))    # of what the first one left


@pytest.mark.parametrize("first,recent", [(0, 10), (4, 0), (3, 20), (50, 50), (0, 1000), (1000, 0), (10, 63)])
def test_first_and_recent(salt_lib, ctx, first, recent):
    c = Cache(salt_lib, ctx, [100, 64, 65, 500], kv_heads=3)
    c.check([64, 64, 64, 64], scores_of(c, "ties"), first, recent)


@pytest.mark.parametrize("kv_heads", [1, 5, 8])
@pytest.mark.parametrize("layer,n_layers", [(0, 1), (1, 2), (3, 1), (2, 0)])
def test_some_layers(salt_lib, ctx, layer, n_layers, kv_heads):
    c = Cache(salt_lib, ctx, [90, 50], kv_heads=kv_heads, layers=4)
    c.check([30, 30], scores_of(c, "normal"), 1, 5, layer, n_layers)


def test_without_weights_and_with_wider_lines(salt_lib, ctx):
    c = Cache(salt_lib, ctx, [90, 50])
    c.check([30, 50], scores_of(c, "normal"), places=70, weights=False)


def test_by_the_weights_themselves(salt_lib, ctx):
    c = Cache(salt_lib, ctx, [90, 50, 2000])
    c.check([30, 45, 700], c.t["weights"], 2, 5)


def test_what_cannot_be_kept(salt_lib, ctx):
    """Fewer than no tokens, or more than a line of places holds: the request stays and the error word says so."""
    c = Cache(salt_lib, ctx, [90, 50, 70])
    c.check([20, -1, 10], scores_of(c, "normal"), flags=0x400)
    c = Cache(salt_lib, ctx, [90, 50, 70])
    c.check([20, 31, 10], scores_of(c, "normal"), places=30, flags=0x400)
    c.check([0, 0, 0], scores_of(c, "normal"))


@pytest.mark.parametrize("n,keep,first,recent,kind", [(5000, 4999, 0, 0, "normal"), (5000, 1, 0, 0, "ties"), (8192, 4096, 4, 512, "normal"),
                                                      (70001, 20000, 0, 1024, "close"), (70001, 69000, 100, 0, "equal"), (33000, 33, 1, 1, "strange")])
@pytest.mark.parametrize("dim,page,kv_heads", [(64, 128, 1), (128, 16, 2)])
def test_long_lines(salt_lib, ctx, n, keep, first, recent, kind, dim, page, kv_heads):
    c = Cache(salt_lib, ctx, [n, 100], dim=dim, page=page, kv_heads=kv_heads, layers=1)
    c.check([keep, 50], scores_of(c, kind), first, recent)


def test_lines_longer_than_shared_memory(salt_lib, ctx):
    """Scores that no cluster's shared memory holds are read again."""
    c = Cache(salt_lib, ctx, [400003, 17], dim=64, page=128, kv_heads=1, layers=1)
    c.check([123456, 17], scores_of(c, "close"), 3, 1000)


def test_many_lines(salt_lib, ctx):
    lens = [int(n) for n in np.random.RandomState(1).randint(1, 200, 300)]
    c = Cache(salt_lib, ctx, lens, kv_heads=4, layers=2)
    c.check([n * 2 // 3 for n in lens], scores_of(c, "normal"), 1, 8)


def test_offsets_past_32_bits(salt_lib, ctx):
    layers, pages, kv_heads, page, dim = 35, 8192, 4, 64, 64
    shape = (layers, pages, kv_heads, page)
    k, v = (torch.zeros(shape + (dim,), dtype=torch.uint8, device="cuda") for _ in range(2))
    e = [torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2)]
    w = torch.zeros(shape, device="cuda")
    kv = salt_lib.salt_kv_create(ctx, k, v, *e)
    plan = salt_lib.salt_attn_create(kv, 4, 1, 1, 4)
    salt_lib.salt_attn_track(plan)
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([1], [130], [0, 3], [8191, 0, 8190]))
    w[-1, 8190, :, :2] = 1.0
    k[-1, 8190, :, 1], v[-1, 8190, :, 0], e[0][-1, 8190, :, 1] = 3, 4, 5
    kept = torch.zeros((1, 1, 4, 2), dtype=torch.int32, device="cuda")
    salt_lib.salt_attn_evict(plan, layers - 1, 1, torch.tensor([2], dtype=torch.int32, device="cuda"), w, kept, weights=w)
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0
    assert bool((kept == torch.tensor([128, 129], device="cuda")).all())
    assert bool((w[-1, 8191, :, :2] == 1).all()) and int(w.sum()) == 16
    assert bool((k[-1, 8191, :, 1] == 3).all()) and bool((v[-1, 8191, :, 0] == 4).all()) and bool((e[0][-1, 8191, :, 1] == 5).all())
    assert int(k.sum(dtype=torch.int64)) == 2 * 4 * 64 * 3


def test_on_another_stream(salt_lib, ctx):
    c = Cache(salt_lib, ctx, [90, 50, 2000])
    c.check([30, 45, 700], scores_of(c, "normal"), 2, 5, stream=torch.cuda.Stream())


def test_captured_and_replayed(salt_lib, ctx):
    """A captured call goes by the build that it is replayed after; one of more requests is left as it is."""
    c = Cache(salt_lib, ctx, [90, 500, 70], layers=1)
    fresh = [c.t[n].clone() for n in ARRAYS]
    scores, keep = scores_of(c, "ties"), torch.tensor([30, 200, 60], dtype=torch.int32, device="cuda")
    kept = torch.full((1, 3, 2, 200), -7, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        salt_lib.salt_attn_evict(c.plan, 0, 1, keep, scores, kept, 0, 8, c.t["weights"])
    for lens in ([90, 500, 70], [40, 490, 70], [90, 500]):
        for n, x in zip(ARRAYS, fresh):
            c.t[n].copy_(x)
        kept.fill_(-7)
        b = dict(c.batch, kv_len=lens, page_ptr=c.batch["page_ptr"][:len(lens) + 1])
        c.build(**b)
        graph.replay()
        torch.cuda.synchronize()
        arrays, want = evict([x.cpu().numpy() for x in fresh], b, 16, [0], keep.tolist()[:len(lens)], scores.cpu().numpy(),
                             np.full((1, len(lens), 2, 200), -7), 0, 8)
        assert np.array_equal(kept.cpu().numpy()[:, :len(lens)], want) and bool((kept[:, len(lens):] == -7).all())
        assert all(np.array_equal(c.t[n].cpu().numpy().view(np.uint8), a.view(np.uint8)) for n, a in zip(ARRAYS, arrays))
    assert salt_lib.salt_get_device_error(ctx) == 0
    small = torch.cuda.CUDAGraph()
    c.build(**dict(c.batch, kv_len=[90, 500], page_ptr=c.batch["page_ptr"][:3]))
    with torch.cuda.graph(small):
        salt_lib.salt_attn_evict(c.plan, 0, 1, keep[:2], scores, kept[:, :2].contiguous(), 0, 8, c.t["weights"])
    c.build()
    before = c.host()
    small.replay()
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0x80
    assert all(np.array_equal(a.view(np.uint8), b.view(np.uint8)) for a, b in zip(before, c.host()))


def test_captured_for_short_lines_and_replayed_on_long_ones(salt_lib, ctx):
    c = Cache(salt_lib, ctx, [9001, 300], layers=1, kv_heads=3, page=64)
    scores, keep = scores_of(c, "normal"), torch.tensor([5000, 100], dtype=torch.int32, device="cuda")
    kept = torch.full((1, 2, 3, 5000), -7, dtype=torch.int32, device="cuda")
    c.build(kv_len=[40, 300])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        salt_lib.salt_attn_evict(c.plan, 0, 1, keep, scores, kept, 1, 9, c.t["weights"])
    c.build()
    before = c.host()
    graph.replay()
    torch.cuda.synchronize()
    arrays, want = evict(before, c.batch, 64, [0], [5000, 100], scores.cpu().numpy(), np.full((1, 2, 3, 5000), -7), 1, 9)
    assert np.array_equal(kept.cpu().numpy(), want) and salt_lib.salt_get_device_error(ctx) == 0
    assert all(np.array_equal(a.view(np.uint8), b.view(np.uint8)) for a, b in zip(c.host(), arrays))


def test_refusals(salt_lib, ctx):
    c = Cache(salt_lib, ctx, [90, 50])
    before = c.host()
    keep, s = torch.tensor([30, 20], dtype=torch.int32, device="cuda"), scores_of(c, "normal")
    kept = torch.full((2, 2, 2, 30), -7, dtype=torch.int32, device="cuda")

    def refused(name, call):
        with pytest.raises(salt_lib.SaltError) as e:
            call()
        assert e.value.name == name, e.value

    run = lambda layer=0, n=2, keep=keep, s=s, kept=kept, plan=None, **kw: salt_lib.salt_attn_evict(plan or c.plan, layer, n, keep, s, kept, **kw)  # noqa: E731
    refused("SALT_ERR_INVALID_ARG", lambda: run(first=-1))
    refused("SALT_ERR_INVALID_ARG", lambda: run(recent=-1))
    refused("SALT_ERR_LAYER_RANGE", lambda: run(layer=1))
    refused("SALT_ERR_LAYER_RANGE", lambda: run(layer=-1))
    odd = torch.zeros(s.numel() + 1, device="cuda")[1:].view(s.shape)
    refused("SALT_ERR_ALIGN", lambda: run(s=odd))
    refused("SALT_ERR_ALIGN", lambda: run(weights=odd))
    for kw in (dict(keep=keep[:1]), dict(keep=keep.long()), dict(s=s.double()), dict(s=s[:1]), dict(kept=kept[:, :1]), dict(kept=kept.long()),
               dict(kept=kept[..., :20]), dict(kept=kept[0]), dict(weights=s.half())):
        with pytest.raises(ValueError):
            run(**kw)
    lib, st = salt_lib._lib, torch.cuda.current_stream().cuda_stream
    for args in ((None, 0, 0, s.data_ptr(), None, kept.data_ptr(), 30), (keep.data_ptr(), 0, 0, None, None, kept.data_ptr(), 30),
                 (keep.data_ptr(), 0, 0, s.data_ptr(), None, None, 30), (keep.data_ptr(), 0, 0, s.data_ptr(), None, kept.data_ptr(), -1)):
        assert lib.salt_attn_evict(c.plan.handle, 0, 2, *args, st) == 1
    plan = salt_lib.salt_attn_create(c.kv, 2, 2, 3, 40)
    refused("SALT_ERR_NOT_BUILT", lambda: salt_lib.salt_attn_evict(plan, 0, 2, keep[:0], s, kept[:, :0]))
    salt_lib.salt_attn_track(plan)
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([1, 1], [20, 20], [0, 2, 4], [0, 1, 2, 1]))
    refused("SALT_ERR_INVALID_ARG", lambda: run(plan=plan))
    torch.cuda.synchronize()
    assert all(np.array_equal(a.view(np.uint8), b.view(np.uint8)) for a, b in zip(before, c.host()))
    assert bool((kept == -7).all()) and salt_lib.salt_get_device_error(ctx) == 0
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([], [], [0], []))
    salt_lib.salt_attn_evict(plan, 0, 2, keep[:0], s, kept[:, :0])


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64)])
def test_a_cache_whose_tokens_come_and_go(salt_lib, ctx, dim, page):
    """Steps of three requests of one layer: keys rotated to their positions into the cache, attention, its
    weights gathered, and every second step the tokens over a budget taken out.  Each
    operator's results are held against its definition on the cache as it was before."""
    salt, heads, kv_heads, budget = salt_lib, 4, 2, 40
    g = torch.Generator().manual_seed(dim)
    freq, scale = frequencies(dim), dim ** -0.5
    prompt, group = 33, [0, -1, 0]
    pages = [[7, 0, 3, 11, 15, 17], [1, 9, 2, 10, 13, 18], [4, 8, 5, 12, 14, 19]] if page == 16 else [[7], [1], [4]]
    pre = [6, 16, 20] if page == 16 else [6]
    n_pages = 21
    shape = (1, n_pages, kv_heads, page, dim)
    byte = dict(dtype=torch.uint8, device="cuda")
    k, v, ke, ve = torch.zeros(shape, **byte), torch.zeros(shape, **byte), torch.zeros(shape[:4], **byte), torch.zeros(shape[:4], **byte)
    w = torch.full(shape[:4], math.nan, device="cuda")
    kv, rope = salt.salt_kv_create(ctx, k, v, ke, ve), salt.salt_rope_create(ctx, dim, dim, freq)
    plan = salt.salt_attn_create(kv, heads, 3, 200, 30, 1)
    salt.salt_attn_track(plan)
    norm = (1.0 + 0.3 * torch.randn(dim, generator=g)).bfloat16()

    def write(positions, slots):
        T = len(positions)
        qkv = torch.randn((T, heads + 2 * kv_heads, dim), generator=g).bfloat16()
        d, q = qkv.cuda(), torch.empty((T, heads, dim), dtype=torch.bfloat16, device="cuda")
        salt.salt_rope_write(rope, kv, 0, d[:, :heads], d[:, heads:heads + kv_heads], d[:, heads + kv_heads:],
                             torch.tensor(positions, dtype=torch.int32, device="cuda"), torch.tensor(slots, dtype=torch.int32, device="cuda"), q,
                             norm.cuda(), norm.cuda())
        check_bf16(q.cpu(), *rotate(qkv[:, :heads], positions, freq, norm=norm))
        return q

    slot = lambda p, j: p[j // page] * page + j % page  # noqa: E731
    write(list(range(prompt)), [slot(pre, j) for j in range(prompt)])
    w[0, torch.tensor(pre)] = 0.0
    cached, position = [0, 0, 0], [prompt, 0, prompt]
    for step, q_len in enumerate([(30, 50, 1), (1, 1, 1), (20, 3, 30), (1, 4, 15)]):
        slots = [slot(pages[b], cached[b] + i) for b in range(3) for i in range(q_len[b])]
        q = write([position[b] + i for b in range(3) for i in range(q_len[b])], slots)
        cached, position = ([x[b] + q_len[b] for b in range(3)] for x in (cached, position))
        batch = dict(q_len=list(q_len), kv_len=list(cached), page_ptr=np.cumsum([0] + [len(p) for p in pages]).tolist(), pages=sum(pages, []),
                     group=group, group_len=[prompt], group_page_ptr=[0, len(pre)], group_pages=pre)
        salt.salt_attn_build(plan, salt.salt_attn_batch(**batch))
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        salt.salt_attn_run(plan, 0, q, out, scale, lse)
        before = w.clone()
        salt.salt_attn_weights(plan, 0, q, lse, scale, w, 0.9)
        torch.cuda.synchronize()
        K, V = value(k[0], ke[0]), value(v[0], ve[0])
        compare(out.cpu(), lse.cpu(), *attention(q.cpu(), K, V, batch, page, scale))
        check_weights(w[0].cpu(), *add_weights(before[0].cpu(), K, q.cpu(), lse.cpu(), batch, page, scale, 0.9))
        if step % 2:
            arrays = [x.cpu().numpy() for x in (k, v, ke, ve, w)]
            kept = torch.full((1, 3, kv_heads, budget), -1, dtype=torch.int32, device="cuda")
            want, places = evict(arrays, batch, page, [0], [budget] * 3, arrays[4], kept.cpu().numpy(), 2, 8)
            salt.salt_attn_evict(plan, 0, 1, torch.full((3,), budget, dtype=torch.int32, device="cuda"), w, kept, 2, 8, w)
            torch.cuda.synchronize()
            for x, y in zip((k, v, ke, ve, w), want):
                assert np.array_equal(x.cpu().numpy().view(np.uint8), y.view(np.uint8))
            assert np.array_equal(kept.cpu().numpy(), places)
            cached = [min(n, budget) for n in cached]
    assert salt.salt_get_device_error(ctx) == 0
