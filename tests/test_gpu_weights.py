"""The cached tokens' attention weights against the 64-bit definition: shapes of
batches, masks that leave rows empty, what lies outside the lists, NaN, order, streams, graphs and
refusals."""
import math

import pytest
import torch

from attn_reference import value
from keeping_reference import add_weights, check_weights
from test_gpu_attn import World

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


class Weights(World):
    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.salt.salt_attn_track(self.plan)
        shape = self.exps["k"].shape
        self.w = torch.exp(torch.randn(shape, generator=torch.Generator().manual_seed(9)))
        k, v = (value(self.codes[n][self.layer], self.exps[n][self.layer]) for n in ("k", "v"))
        self.k_values = k
        if not hasattr(self, "lse"):
            self.lse = self.reference()[1].float()

    def weights(self, decay=1.0, q=None, lse=None, stream=None):
        """Of the whole cache, between guard values."""
        n = self.w.numel()
        buf = torch.full((n + 64,), 7.0, device="cuda")
        w = buf[32:32 + n].view(self.w.shape)
        w.copy_(self.w)
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.salt.salt_attn_weights(self.plan, self.layer, self.q.cuda() if q is None else q, (self.lse if lse is None else lse).cuda(),
                                    self.scale, w, decay, stream)
        torch.cuda.synchronize()
        assert bool((buf[:32] == 7).all()) and bool((buf[-32:] == 7).all()) and self.salt.salt_get_device_error(self.ctx) == 0
        return w.cpu()

    def check(self, decay=1.0, **kw):
        got = self.weights(decay, **kw)
        q, lse = (kw.get(n, x).cpu() for n, x in (("q", self.q), ("lse", self.lse)))
        want, tol = add_weights(self.w[self.layer], self.k_values, q, lse, self.batch, self.page, self.scale, decay)
        check_weights(got[self.layer], want, tol)
        others = [l for l in range(got.shape[0]) if l != self.layer]
        assert torch.equal(got[others], self.w[others])
        return got


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv", [0, 1, 2, 16, 17, 127, 128, 129, 300])
def test_one_token_of_one_request(salt_lib, ctx, kv, dim):
    w = Weights(salt_lib, ctx, [1], [kv], dim=dim, seed=kv)
    w.build()
    w.check()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (8, 2), (12, 4), (40, 5), (64, 1)])
def test_ragged_batch(salt_lib, ctx, page, dim, heads, kv_heads):
    """Decode, drafts and short prompts together, groups used by many, one and no request, empty
    requests, more query than cached tokens."""
    w = Weights(salt_lib, ctx, [1, 3, 0, 5, 1, 20, 1, 2], [40, 7, 30, 3, 0, 133, 1, 260], [0, 0, 1, 2, -1, 2, 0, -1], [150, 33, 16, 77, 0],
                heads=heads, kv_heads=kv_heads, dim=dim, page=page, layers=2, layer=1, seed=heads + dim)
    w.build()
    w.check(0.75)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,kv,prompt,heads,kv_heads", [(129, 129, 0, 4, 2), (200, 333, 100, 4, 1), (70, 70, 300, 5, 1), (300, 150, 40, 2, 2),
                                                        (17, 400, 0, 16, 1), (40, 500, 130, 6, 2)])
def test_prompt_chunks(salt_lib, ctx, n, kv, prompt, heads, kv_heads, dim):
    w = Weights(salt_lib, ctx, [n, 1, n // 2], [kv, 5, kv], [0, 0, 0] if prompt else None, [prompt] if prompt else (), heads=heads,
                kv_heads=kv_heads, dim=dim, page=32, seed=n)
    w.build()
    w.check()


@pytest.mark.parametrize("q_len,kv_len,group,group_len", [([1] * 70, [20 + i for i in range(70)], [i % 2 for i in range(70)], [140, 90]),
                                                          ([3] * 40, [9] * 40, [0] * 40, [260])])
def test_many_requests(salt_lib, ctx, q_len, kv_len, group, group_len):
    w = Weights(salt_lib, ctx, q_len, kv_len, group, group_len, heads=8, kv_heads=2, dim=64, page=16)
    w.build()
    w.check(0.9)


@pytest.mark.parametrize("decay", [0.0, 0.5, -1.0])
def test_what_was_there(salt_lib, ctx, decay):
    """With no decay, and for the step's own tokens, what was there is not read; tokens that no row sees keep it."""
    w = Weights(salt_lib, ctx, [4, 2, 0], [30, 2, 10], [0, 0, 1], [40, 20], dim=128)
    b = w.batch
    new = lambda i, j: (0, b["pages"][b["page_ptr"][i] + j // 16], slice(None), j % 16)  # noqa: E731
    for i, j in ((0, 26), (0, 29), (1, 0), (1, 1)):
        w.w[new(i, j)] = math.nan
    if decay == 0.0:
        w.w[new(0, 0)] = math.inf
        w.w[0, b["group_pages"][0]] = math.nan
    w.build()
    got = w.check(decay)
    idle = b["pages"][b["page_ptr"][2]]
    assert torch.equal(got[0, idle], w.w[0, idle])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [2, 90])
def test_nan(salt_lib, ctx, dim, n):
    """A key that stands for NaN spoils its token's weight; a NaN in a row's query or log-sum those that the row
    sees; an infinity in its query too, by the log-sum that the attention leaves; rows that see nothing spoil none."""
    def world():
        return Weights(salt_lib, ctx, [n, 3], [n + 40, 2], [0, -1], [50], heads=4, kv_heads=2, dim=dim, page=16, seed=n)
    w = world()
    b = w.batch
    w.q[n] = math.nan          # sees nothing: three query tokens, two cached
    w.lse[n] = math.nan
    e = w.exps["k"]
    e[0, b["pages"][0], 1, 3] = 255
    w.codes["k"][0, b["pages"][0], 1, 3] = 0
    w.k_values = value(w.codes["k"][0], w.exps["k"][0])
    w.build()
    got = w.check()
    assert int(got.isnan().sum()) == 1
    for what in ("q", "inf", "lse"):
        w = world()
        if what == "q":
            w.q[1, 2, 5] = math.nan
        elif what == "inf":
            w.q[1, 2, 5] = -math.inf
            w.build()
            w.lse = w.run()[1]
        else:
            w.lse[1, 2] = math.nan
        w.build()
        got = w.weights()
        want = add_weights(w.w[0], w.k_values, w.q, w.lse, w.batch, 16, w.scale, 1.0)[0]
        j = torch.arange(42)   # tokens that row 1 sees: 40 + 2 of its own, the prompt's 50
        spoiled = torch.zeros_like(got[0], dtype=torch.bool)
        spoiled[torch.tensor(b["pages"])[j // 16], 1, j % 16] = True
        j = torch.arange(50)
        spoiled[torch.tensor(b["group_pages"])[j // 16], 1, j % 16] = True
        assert torch.equal(got[0].isnan(), spoiled) and torch.equal(want.isnan(), spoiled) and not bool(got.isinf().any())


def test_of_the_attention_itself(salt_lib, ctx):
    """With the log-sums that a run leaves, each row gives one in all, for each of its heads."""
    w = Weights(salt_lib, ctx, [1, 5, 60, 1], [90, 5, 200, 0], [0, 0, -1, 0], [170], heads=8, kv_heads=2, dim=128, page=64)
    w.build()
    _, lse = w.run()
    w.w.zero_()
    got = w.check(lse=lse)
    assert torch.allclose(got.double().sum((0, 1, 3)), torch.tensor([67.0 * 4] * 2, dtype=torch.float64), rtol=2.0 ** -14)
    assert torch.equal(got, w.weights(lse=lse))


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(salt_lib, ctx, scale):
    w = World(salt_lib, ctx, [1, 30], [60, 30], dim=64)
    w.scale = scale
    lse = w.reference()[1].float()
    w = Weights(salt_lib, ctx, [1, 30], [60, 30], dim=64)
    w.scale, w.lse = scale, lse
    w.build()
    w.check()


def test_strided_queries(salt_lib, ctx):
    w = Weights(salt_lib, ctx, [1, 40], [70, 40], [0, 0], [33], heads=4, kv_heads=2, dim=64)
    w.build()
    fused = torch.randn((41, 7 * 64)).bfloat16().cuda()
    q = fused[:, 64:5 * 64].unflatten(1, (4, 64))
    q.copy_(w.q)
    assert torch.equal(w.weights(q=q), w.weights())


def test_spread_of_queries(salt_lib, ctx):
    """Elements far below their row's largest count as they should."""
    w = Weights(salt_lib, ctx, [1, 20], [100, 120], heads=4, kv_heads=1, dim=128)
    w.q[..., 0] *= 2.0 ** 10
    w.q[3] *= 2.0 ** -40
    w.q[4, 1] = 0.0
    w.lse = w.reference()[1].float()
    w.build()
    w.check()


@pytest.mark.parametrize("dim,kv_heads", [(64, 2), (128, 1)])
def test_long(salt_lib, ctx, dim, kv_heads):
    """Ranges that go over many tiles of every CTA, by sums over them: uniform queries of zeros give each token what they should."""
    n, page = 200001, 64
    pages = -(-n // page)
    shape = (1, pages, kv_heads, page, dim)
    t = [torch.randint(0, 0x70, shape, dtype=torch.uint8, device="cuda") for _ in range(2)]
    e = [torch.full(shape[:4], 120, dtype=torch.uint8, device="cuda") for _ in range(2)]
    kv = salt_lib.salt_kv_create(ctx, t[0], t[1], e[0], e[1])
    plan = salt_lib.salt_attn_create(kv, 4 * kv_heads, 1, 3, pages)
    salt_lib.salt_attn_track(plan)
    order = torch.randperm(pages).tolist()
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([3], [n], [0, pages], order))
    q = torch.randn((3, 4 * kv_heads, dim), device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((3, 4 * kv_heads), device="cuda")
    salt_lib.salt_attn_run(plan, 0, q, out, dim ** -0.5, lse)
    w = torch.ones(shape[:4], device="cuda")
    salt_lib.salt_attn_weights(plan, 0, q, lse, dim ** -0.5, w, 1.0)
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0
    K = t[0][0].view(torch.float8_e4m3fn).double() * 2.0 ** -7                                        # [pages, KV, page, D]
    K = K[torch.tensor(order, device="cuda")].transpose(1, 2).reshape(-1, kv_heads, dim)[:n]
    x = q.double().view(3, kv_heads, 4, dim)
    s = torch.einsum("rkgd,nkd->kngr", x, K) * dim ** -0.5
    see = torch.arange(n, device="cuda")[:, None] < torch.tensor([n - 2, n - 1, n], device="cuda")
    p = torch.exp(s - lse.double().view(3, kv_heads, 4).permute(1, 2, 0)[:, None]) * see[None, :, None]
    want = p.sum((2, 3)).T
    want[:n - 3] += 1.0
    got = w[0][torch.tensor(order, device="cuda")].transpose(1, 2).reshape(-1, kv_heads)
    assert bool((got[n:] == 1.0).all())
    # (scores below 2^5 with sums of |q k| below 2^9: by add_weights' bound under 2^-9 of the new part, 2^-22 of the rest)
    assert bool(((got[:n].double() - want).abs() <= (want - 1.0).abs() * 2.0 ** -9 + 2.0 ** -22).all())


def test_offsets_past_32_bits(salt_lib, ctx):
    """The last layer of a cache of more than 2^32 bytes of codes."""
    layers, pages, kv_heads, page, dim = 35, 8192, 4, 64, 64
    shape = (layers, pages, kv_heads, page, dim)
    k = torch.zeros(shape, dtype=torch.uint8, device="cuda")
    v = k  # (not read)
    e = torch.zeros(shape[:4], dtype=torch.uint8, device="cuda")
    kv = salt_lib.salt_kv_create(ctx, k, v, e, e)
    plan = salt_lib.salt_attn_create(kv, 4, 1, 1, 4)
    salt_lib.salt_attn_track(plan)
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([1], [130], [0, 3], [8191, 0, 8190]))
    k[-1, 8190] = 0x38                                          # ones
    e[-1, 8190] = 127
    w = torch.zeros(shape[:4], device="cuda")
    q, lse = torch.ones((1, 4, dim), dtype=torch.bfloat16, device="cuda"), torch.full((1, 4), 60.0, device="cuda")
    salt_lib.salt_attn_weights(plan, layers - 1, q, lse, 1.0, w)
    torch.cuda.synchronize()
    want = torch.zeros((3, 64), dtype=torch.float64)
    want[:2], want[2, :2] = math.exp(-60.0), math.exp(4.0)
    got = w[-1, torch.tensor([8191, 0, 8190], device="cuda")].double().cpu()
    assert bool(((got - want[:, None]).abs() <= want[:, None] * 2.0 ** -15).all())
    assert int((w != 0).sum()) == 130 * 4


def test_other_stream_and_order(salt_lib, ctx):
    w = Weights(salt_lib, ctx, [1, 40], [70, 40], [0, 0], [33], heads=4, kv_heads=2, dim=64)
    w.build()
    a = w.weights()
    assert torch.equal(a, w.weights(stream=torch.cuda.Stream()))
    assert torch.equal(a, w.weights())


def test_captured_and_replayed(salt_lib, ctx):
    """A captured call replays on a later build of at most as many query tokens; on a larger one it does nothing and says so."""
    big = Weights(salt_lib, ctx, [2, 40], [70, 60], [0, 0], [200], heads=4, kv_heads=2, dim=64)
    w = big.w.cuda()
    q, lse = big.q.cuda(), big.lse.cuda()
    small = dict(big.batch, q_len=[1, 30], kv_len=[66, 60])
    def build(b):
        salt_lib.salt_attn_build(big.plan, salt_lib.salt_attn_batch(b["q_len"], b["kv_len"], b["page_ptr"], b["pages"], b["group"],
                                                                    b["group_len"], b["group_page_ptr"], b["group_pages"]))
    def replayed(graph, batch):
        w.copy_(big.w)
        graph.replay()
        torch.cuda.synchronize()
        want, tol = add_weights(big.w[0], big.k_values, big.q, big.lse, batch, 16, big.scale, 0.5)
        check_weights(w[0].cpu(), want, tol)
    graphs = []
    for b in (big.batch, small):
        build(b)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            salt_lib.salt_attn_weights(big.plan, 0, q, lse, big.scale, w, 0.5)
    build(big.batch)
    replayed(graphs[0], big.batch)
    w.copy_(big.w)
    graphs[1].replay()
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0x80 and torch.equal(w.cpu(), big.w)
    build(small)
    replayed(graphs[0], small)
    replayed(graphs[1], small)
    assert salt_lib.salt_get_device_error(ctx) == 0


def test_captured_for_one_kind_of_lists_and_replayed_on_others(salt_lib, ctx):
    """Single tokens, long chunks and both, each captured and replayed on the others."""
    big = Weights(salt_lib, ctx, [120, 1, 3], [300, 70, 5], [0, -1, 0], [200], heads=4, kv_heads=2, dim=64)
    batches = [big.batch, dict(big.batch, q_len=[1, 1, 3], kv_len=[200, 70, 5]), dict(big.batch, q_len=[120, 0, 0])]
    w, q, lse = big.w.cuda(), big.q.cuda(), big.lse.cuda()
    graphs = []

    def build(b):
        salt_lib.salt_attn_build(big.plan, salt_lib.salt_attn_batch(b["q_len"], b["kv_len"], b["page_ptr"], b["pages"], b["group"], b["group_len"],
                                                                    b["group_page_ptr"], b["group_pages"]))
    for b in batches:
        build(b)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            salt_lib.salt_attn_weights(big.plan, 0, q, lse, big.scale, w, 0.5)
    for i, g in enumerate(graphs):
        for b in batches:
            build(b)
            w.copy_(big.w)
            g.replay()
            torch.cuda.synchronize()
            if sum(b["q_len"]) > sum(batches[i]["q_len"]):
                assert salt_lib.salt_get_device_error(ctx) == 0x80 and torch.equal(w.cpu(), big.w)
                continue
            assert salt_lib.salt_get_device_error(ctx) == 0
            T = sum(b["q_len"])
            want, tol = add_weights(big.w[0], big.k_values, big.q[:T], big.lse[:T], b, 16, big.scale, 0.5)
            # (log-sums of another batch: their exponentials may pass fp32's range)
            fine = want.abs() < 1e30
            got = w[0].cpu().double()
            assert bool(((got - want).abs() <= tol)[fine].all())


def test_refusals(salt_lib, ctx):
    w = Weights(salt_lib, ctx, [1, 2], [20, 30], dim=64)
    q, lse, x = w.q.cuda(), w.lse.cuda(), w.w.cuda()

    def refused(name, call):
        with pytest.raises(salt_lib.SaltError) as e:
            call()
        assert e.value.name == name, e.value

    run = lambda layer=0, q=q, lse=lse, scale=0.1, x=x, decay=1.0: salt_lib.salt_attn_weights(w.plan, layer, q, lse, scale, x, decay)  # noqa: E731
    refused("SALT_ERR_NOT_BUILT", run)
    w.build()
    run()
    torch.cuda.synchronize()
    before = x.clone()
    refused("SALT_ERR_LAYER_RANGE", lambda: run(layer=1))
    refused("SALT_ERR_LAYER_RANGE", lambda: run(layer=-1))
    refused("SALT_ERR_INVALID_ARG", lambda: run(scale=math.nan))
    refused("SALT_ERR_INVALID_ARG", lambda: run(decay=math.inf))
    odd = torch.zeros(q.numel() + 4, dtype=torch.bfloat16, device="cuda")[4:].view(q.shape)
    refused("SALT_ERR_ALIGN", lambda: run(q=odd))
    refused("SALT_ERR_ALIGN", lambda: run(x=torch.zeros(x.numel() + 1, device="cuda")[1:].view(x.shape)))
    for kw in (dict(q=q[:2]), dict(q=q.float()), dict(lse=lse[:2]), dict(lse=lse.double()), dict(x=x.double()), dict(x=x[:, :2]), dict(x=x.cpu()),
               dict(q=q[:, :4])):
        with pytest.raises(ValueError):
            run(**kw)
    lib, s = salt_lib._lib, torch.cuda.current_stream().cuda_stream
    for args in ((None, 512, lse.data_ptr()), (q.data_ptr(), 504, lse.data_ptr()), (q.data_ptr(), 512, None)):
        assert lib.salt_attn_weights(w.plan.handle, 0, *args, 0.1, 1.0, x.data_ptr(), s) == 1
    assert lib.salt_attn_weights(w.plan.handle, 0, q.data_ptr(), 512, lse.data_ptr(), 0.1, 1.0, None, s) == 1
    # a plan that was built before it was tracked
    plan = salt_lib.salt_attn_create(w.kv, 8, 2, 3, 10)
    salt_lib.salt_attn_build(plan, w.host_batch())
    salt_lib.salt_attn_track(plan)
    salt_lib.salt_attn_track(plan)
    refused("SALT_ERR_NOT_BUILT", lambda: salt_lib.salt_attn_weights(plan, 0, q, lse, 0.1, x))
    # a page listed twice: by two requests, by one, by a request and a group
    for batch in (([1, 1], [4, 4], [0, 1, 2], [3, 3]), ([1, 1], [4, 30], [0, 1, 3], [0, 1, 1]),
                  ([1, 1], [4, 4], [0, 1, 2], [0, 3], [0, -1], [5], [0, 1], [3])):
        plan = salt_lib.salt_attn_create(w.kv, 8, 2, 3, 10, 1)
        salt_lib.salt_attn_track(plan)
        salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch(*batch))
        out = torch.zeros_like(q)
        salt_lib.salt_attn_run(plan, 0, q, out, 0.1)       # attention may share pages
        refused("SALT_ERR_INVALID_ARG", lambda: salt_lib.salt_attn_weights(plan, 0, q, lse, 0.1, x))
    # pages past the lengths may be anyone's
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([1, 1], [4, 4], [0, 2, 3], [0, 3, 3]))
    salt_lib.salt_attn_weights(plan, 0, q, lse, 0.1, before.clone())
    torch.cuda.synchronize()
    assert torch.equal(x, before)
    # no rows, no requests
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([0, 0], [4, 4], [0, 1, 2], [0, 3]))
    salt_lib.salt_attn_weights(plan, 0, q, lse, 0.1, x)
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([], [], [0], []))
    salt_lib.salt_attn_weights(plan, 0, q[:0], lse[:0], 0.1, x)
    torch.cuda.synchronize()
    assert torch.equal(x, before) and salt_lib.salt_get_device_error(ctx) == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,kv,prompt,heads,kv_heads", [(700, 900, 0, 8, 1), (1500, 1500, 300, 2, 2), (333, 5000, 64, 3, 1), (80, 300, 140000, 8, 8)])
def test_rows_of_a_tile_split(salt_lib, ctx, n, kv, prompt, heads, kv_heads, dim):
    """Few tiles of many rows: parts of a unit's rows meet, the same each time; and more tiles than a build lists. On the GPU in 64 bits."""
    page = 64
    lens = [prompt, kv]
    need = [-(-x // page) for x in lens]
    order = torch.randperm(sum(need) + 1).tolist()
    shape = (1, len(order), kv_heads, page, dim)
    k = torch.randint(0, 0x70, shape, dtype=torch.uint8, device="cuda") | (torch.rand(shape, device="cuda") < 0.5).to(torch.uint8) * 128
    e = torch.randint(117, 121, shape[:4], dtype=torch.uint8, device="cuda")
    cache = salt_lib.salt_kv_create(ctx, k, k, e, e)
    plan = salt_lib.salt_attn_create(cache, heads, 1, n, sum(need), 1)
    salt_lib.salt_attn_track(plan)
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch([n], [kv], [0, need[1]], order[need[0]:sum(need)], [0], [prompt], [0, need[0]], order[:need[0]]))
    q = torch.randn((n, heads, dim), device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((n, heads), device="cuda")
    salt_lib.salt_attn_run(plan, 0, q, out, dim ** -0.5, lse)
    w = torch.full(shape[:4], 0.5, device="cuda")
    w[0, order[-1]] = math.nan   # not in the batch
    first = w.clone()
    salt_lib.salt_attn_weights(plan, 0, q, lse, dim ** -0.5, first, 0.5)
    for _ in range(3):
        again = w.clone()
        salt_lib.salt_attn_weights(plan, 0, q, lse, dim ** -0.5, again, 0.5)
        assert torch.equal(again[0, order[:-1]], first[0, order[:-1]])
    assert salt_lib.salt_get_device_error(ctx) == 0 and bool(first[0, order[-1]].isnan().all())
    K = k[0].view(torch.float8_e4m3fn).double() * torch.exp2(e[0].double() - 127)[..., None]
    x = q.double().view(n, kv_heads, heads // kv_heads, dim)
    ls = lse.double().view(n, kv_heads, -1).permute(1, 2, 0)[:, None]
    for own in (False, True):
        m, pages = (kv, order[need[0]:sum(need)]) if own else (prompt, order[:need[0]])
        if m == 0:
            continue
        Kl = K[torch.tensor(pages, device="cuda")].transpose(1, 2).reshape(-1, kv_heads, dim)[:m]
        s = torch.einsum("rkgd,nkd->kngr", x, Kl) * dim ** -0.5
        j = torch.arange(m, device="cuda")
        see = j[:, None] <= kv - n + torch.arange(n, device="cuda") if own else torch.ones((m, n), dtype=torch.bool, device="cuda")
        p = torch.exp(s - ls) * see[None, :, None]
        ds = (Kl.abs().sum(-1).T[:, :, None, None] * x.abs().amax(-1).permute(1, 2, 0)[:, None] * 2.0 ** -22
              + torch.einsum("rkgd,nkd->kngr", x.abs(), Kl.abs()) * dim * 2.0 ** -23) * dim ** -0.5 + (s.abs() + ls.abs()) * 2.0 ** -21 + 2.0 ** -20
        tol = (p * (torch.expm1(ds) + n * heads // kv_heads * 2.0 ** -24)).sum((2, 3)).T + 2.0 ** -22
        want = p.sum((2, 3)).T + torch.where((j < kv - n)[:, None] if own else torch.ones((m, 1), dtype=torch.bool, device="cuda"), 0.25, 0.0)
        got = first[0][torch.tensor(pages, device="cuda")].transpose(1, 2).reshape(-1, kv_heads)
        assert bool(((got[:m].double() - want).abs() <= tol).all())
        assert bool((got[m:] == 0.5).all())
