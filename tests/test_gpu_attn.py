"""Attention over the paged 8-bit cache against the 64-bit definition: lengths
from none to long, ragged groups, masks that leave rows empty, stale and
non-finite memory past the lengths, strides, streams, graphs and refusals.

The caches hold what the 64-bit side reads too, so quantisation is no part of
the difference; the tolerance of each element is derived in attn_reference.
"""
import numpy as np
import pytest
import torch

from attn_reference import attention, quantise, value

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


class World:
    """A cache with a batch's tokens in it, the rest of its pages holding NaN
    codes and wild exponents, and the batch's query."""

    def __init__(self, salt, ctx, q_len, kv_len, group=None, group_len=(), heads=8, kv_heads=2, dim=64, page=16, layers=1,
                 layer=0, seed=0, spread=1.0, q_scale=1.0, v_scale=1.0):
        self.salt, self.ctx = salt, ctx
        self.heads, self.kv_heads, self.dim, self.page, self.layer = heads, kv_heads, dim, page, layer
        g = torch.Generator().manual_seed(seed)
        r = np.random.RandomState(seed)
        group = [-1] * len(q_len) if group is None else list(group)
        need = [-(-n // page) for n in list(group_len) + list(kv_len)]
        n_pages = sum(need) + 3
        order = r.permutation(n_pages).tolist()
        lists, ptrs = [], []
        for part in (need[:len(group_len)], need[len(group_len):]):
            ptr, pages = [0], []
            for k in part:
                pages += [order.pop() for _ in range(k)]
                ptr.append(len(pages))
            lists.append(pages)
            ptrs.append(ptr)
        self.batch = dict(q_len=list(q_len), kv_len=list(kv_len), page_ptr=ptrs[1], pages=lists[1], group=group,
                          group_len=list(group_len), group_page_ptr=ptrs[0], group_pages=lists[0])
        self.T = sum(q_len)
        shape = (layers, n_pages, kv_heads, page, dim)
        self.codes, self.exps = {}, {}
        for name in ("k", "v"):
            c = torch.full(shape, 0x7F, dtype=torch.uint8)
            e = torch.full(shape[:4], 254 if name == "k" else 255, dtype=torch.uint8)
            for pages, ptr, lens in ((lists[0], ptrs[0], group_len), (lists[1], ptrs[1], kv_len)):
                for i, n in enumerate(lens):
                    x = torch.randn((n, kv_heads, dim), generator=g) * torch.exp(spread * torch.randn((n, kv_heads, 1), generator=g))
                    x = (x * (v_scale if name == "v" else 1.0)).bfloat16()
                    qc, qe = quantise(x)
                    for j in range(n):
                        p, o = pages[ptr[i] + j // page], j % page
                        c[layer, p, :, o] = qc[j].to(torch.float8_e4m3fn).view(torch.uint8)
                        e[layer, p, :, o] = qe[j].to(torch.uint8)
            self.codes[name], self.exps[name] = c.cuda(), e.cuda()
        self.q = (q_scale * torch.randn((self.T, heads, dim), generator=g)).bfloat16()
        self.scale = dim ** -0.5
        self.kv = salt.salt_kv_create(ctx, self.codes["k"], self.codes["v"], self.exps["k"], self.exps["v"])
        self.plan = salt.salt_attn_create(self.kv, heads, max(1, len(q_len)), max(1, self.T), max(1, len(lists[0]) + len(lists[1])),
                                          len(group_len))

    def host_batch(self):
        b = self.batch
        return self.salt.salt_attn_batch(b["q_len"], b["kv_len"], b["page_ptr"], b["pages"], b["group"], b["group_len"],
                                         b["group_page_ptr"], b["group_pages"])

    def build(self, stream=None):
        self.salt.salt_attn_build(self.plan, self.host_batch(), stream)

    def run(self, q=None, stream=None):
        """out and lse, both between guard rows."""
        q = self.q.cuda() if q is None else q
        buf = torch.full((self.T + 2, self.heads, self.dim), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.T + 2, self.heads), 7.0, device="cuda")
        self.salt.salt_attn_run(self.plan, self.layer, q, buf[1:self.T + 1], self.scale, lse[1:self.T + 1], stream)
        torch.cuda.synchronize()
        assert bool((buf[0] == 7).all()) and bool((buf[-1] == 7).all()) and bool((lse[0] == 7).all()) and bool((lse[-1] == 7).all())
        assert self.salt.salt_get_device_error(self.ctx) == 0
        return buf[1:self.T + 1].cpu(), lse[1:self.T + 1].cpu()

    def reference(self, q=None):
        k, v = (value(self.codes[n][self.layer], self.exps[n][self.layer]) for n in ("k", "v"))
        return attention(self.q if q is None else q.cpu(), k, v, self.batch, self.page, self.scale)

    def check(self, q=None):
        got, glse = self.run(q=q)
        out, lse, tol, ltol = self.reference(q)
        compare(got, glse, out, lse, tol, ltol)
        return got, glse


def compare(got, glse, out, lse, tol, ltol):
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(glse), empty) and bool((glse[empty] < 0).all())
    assert bool((got[empty] == 0).all())
    err = (got.double() - out).abs() - tol
    assert bool((err <= 0).all()), f"out off by {float(err.max()):.3g} over its bound"
    lerr = torch.where(empty, torch.zeros_like(lse), (glse.double() - lse).abs() - ltol)
    assert bool((lerr <= 0).all()), f"lse off by {float(lerr.max()):.3g} over its bound"


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv", [0, 1, 2, 15, 16, 17, 127, 128, 129, 300])
def test_one_token_of_one_request(salt_lib, ctx, kv, dim):
    w = World(salt_lib, ctx, [1], [kv], dim=dim, seed=kv)
    w.build()
    w.check()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (3, 1), (8, 2), (12, 4), (40, 5), (64, 1)])
def test_heads_and_pages(salt_lib, ctx, heads, kv_heads, dim, page):
    w = World(salt_lib, ctx, [1, 3, 0, 2], [140, 3, 50, 77], [0, 1, 0, -1], [200, 33], heads=heads, kv_heads=kv_heads, dim=dim,
              page=page, layers=2, layer=1, seed=heads)
    w.build()
    w.check()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_len,kv_len", [([5], [5]), ([16], [40]), ([33], [33]), ([128], [128]), ([130], [400]), ([257, 1, 64], [257, 300, 129])])
def test_prompt_chunks(salt_lib, ctx, q_len, kv_len, dim):
    w = World(salt_lib, ctx, q_len, kv_len, heads=4, kv_heads=2, dim=dim, page=32, seed=sum(q_len))
    w.build()
    w.check()


@pytest.mark.parametrize("n", [1, 2, 7, 40, 130])
@pytest.mark.parametrize("dim", [64, 128])
def test_shared_prompts(salt_lib, ctx, n, dim):
    """Requests of three groups in no order, a group without requests, one of
    one token, one whose prompt is empty."""
    r = np.random.RandomState(n)
    group = r.choice([-1, 0, 1, 3, 4], n).tolist()
    w = World(salt_lib, ctx, [1] * n, r.randint(0, 40, n).tolist(), group, [260, 1, 90, 0, 128], heads=4, kv_heads=2, dim=dim, page=16,
              seed=n)
    w.build()
    w.check()


def test_rows_that_see_nothing(salt_lib, ctx):
    """Fewer cached tokens than query tokens, none at all, an empty prompt."""
    w = World(salt_lib, ctx, [4, 1, 2, 3], [2, 0, 0, 1], [-1, -1, 0, 1], [0, 5], heads=4, kv_heads=2, dim=128, seed=3)
    w.build()
    got, lse = w.check()
    assert bool(torch.isinf(lse[:2]).all()) and not bool(torch.isinf(lse[2:4]).any()) and bool(torch.isinf(lse[4:7]).all())


def test_no_requests_and_no_tokens(salt_lib, ctx):
    w = World(salt_lib, ctx, [0, 0], [20, 0], heads=4, kv_heads=2)
    w.build()
    w.run()
    salt_lib.salt_attn_build(w.plan, salt_lib.salt_attn_batch([], [], [0], []))
    w.run()


@pytest.mark.parametrize("dim", [64, 128])
def test_scores_far_apart(salt_lib, ctx, dim):
    """Large scores: one token takes nearly everything; and a maximum that
    keeps growing along the cache."""
    w = World(salt_lib, ctx, [2, 1], [700, 513], [0, 0], [900], heads=8, kv_heads=2, dim=dim, q_scale=12.0, seed=5)
    w.build()
    w.check()
    for i in range(w.batch["kv_len"][0]):  # keys' exponents growing with the position
        p, o = w.batch["pages"][i // w.page], i % w.page
        w.exps["k"][0, p, :, o] = 112 + i // 64
    w.check()


@pytest.mark.parametrize("q_scale,v_scale", [(1e-20, 1.0), (1.0, 1e-30), (1.0, 1e30), (0.0, 1.0), (1e-3, 1e-36)])
def test_values_far_from_one(salt_lib, ctx, q_scale, v_scale):
    w = World(salt_lib, ctx, [2], [300], heads=4, kv_heads=2, dim=64, q_scale=q_scale, v_scale=v_scale, seed=8)
    w.build()
    w.check()


def test_values_of_very_different_rows(salt_lib, ctx):
    """Rows of values over 24 binades, rows of zeros among them, and query
    rows whose elements span as many."""
    w = World(salt_lib, ctx, [3], [400], heads=4, kv_heads=2, dim=128, seed=9)
    r = torch.Generator().manual_seed(1)
    w.exps["v"][0] = torch.randint(112, 136, w.exps["v"][0].shape, generator=r).to(torch.uint8).cuda()
    for i in range(0, 400, 7):
        p, o = w.batch["pages"][i // w.page], i % w.page
        w.exps["v"][0, p, :, o] = 0
        w.codes["v"][0, p, :, o] = 0
    w.q = (w.q.float() * torch.exp2(torch.randint(-12, 12, w.q.shape, generator=r).float())).bfloat16()
    w.build()
    w.check()


def test_equal_keys_behind_one_large_score(salt_lib, ctx):
    """One token whose score is 9.5 above many equal ones, which share half of
    the probability: their rounding has one sign and does not average out."""
    w = World(salt_lib, ctx, [1], [6000], heads=4, kv_heads=1, dim=64, page=128, spread=0.0, seed=4)
    first = (w.batch["pages"][0], 0)
    one = torch.zeros(64)
    one[0] = 1.0
    c, e = quantise(one.bfloat16()[None])
    w.codes["k"][0] = c[0].to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    w.exps["k"][0] = int(e[0])
    c, e = quantise((9.5 * one).bfloat16()[None])
    w.codes["k"][0, first[0], 0, 0] = c[0].to(torch.float8_e4m3fn).view(torch.uint8).cuda()
    w.exps["k"][0, first[0], 0, 0] = int(e[0])
    w.q[:] = 0
    w.q[:, :, 0] = torch.tensor([8.0, 8.5, 9.0, 7.5]).bfloat16()
    w.build()
    w.check()


def test_infinities_and_nan(salt_lib, ctx):
    """A cached NaN row spoils the rows that see it and no other; so does a
    query row that is not finite."""
    w = World(salt_lib, ctx, [4, 2], [100, 90], [0, -1], [40], heads=4, kv_heads=2, dim=64, page=16, seed=6)
    at = lambda j: (w.batch["pages"][j // 16], j % 16)  # noqa: E731
    w.exps["k"][0, at(98)[0], 0, at(98)[1]] = 255   # request 0, seen by its query tokens 2 and 3, key head 0
    w.exps["v"][0, at(99)[0], 1, at(99)[1]] = 255   # seen by its query token 3, head 1
    w.build()
    q = w.q.clone()
    q[4, 1, 5] = float("inf")
    q[5, 2, 0] = float("nan")
    got, _ = w.run(q=q.cuda())
    out, lse, tol, ltol = w.reference(q)
    nan = torch.zeros((6, 4), dtype=torch.bool)
    nan[2:4, 0:2] = True
    nan[3, 2:4] = True
    nan[4, 1] = True
    nan[5, 2] = True
    assert bool(torch.isnan(got[nan]).all())
    assert bool(((got.double() - out).abs() <= tol)[~nan].all())


def test_stale_memory_is_never_used(salt_lib, ctx):
    """The result does not depend on what pages hold past the lengths."""
    w = World(salt_lib, ctx, [1, 2, 3], [33, 140, 3], [0, -1, 0], [150], heads=8, kv_heads=2, dim=128, page=64, seed=7)
    w.build()
    a, la = w.run()
    live = {}
    for pages, ptr, lens in ((w.batch["group_pages"], w.batch["group_page_ptr"], w.batch["group_len"]),
                             (w.batch["pages"], w.batch["page_ptr"], w.batch["kv_len"])):
        for i, n in enumerate(lens):
            for j in range(n):
                live.setdefault(pages[ptr[i] + j // 64], []).append(j % 64)
    for name in ("k", "v"):
        c, e = torch.randint(0, 255, w.codes[name].shape, dtype=torch.uint8), torch.randint(0, 255, w.exps[name].shape, dtype=torch.uint8)
        oc, oe = w.codes[name].cpu(), w.exps[name].cpu()
        for p, o in live.items():
            c[0, p][:, o] = oc[0, p][:, o]
            e[0, p][:, o] = oe[0, p][:, o]
        w.codes[name].copy_(c)
        w.exps[name].copy_(e)
    b, lb = w.run()
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_same_bits_each_time_and_beside_other_requests(salt_lib, ctx):
    """Runs repeat bit for bit."""
    w = World(salt_lib, ctx, [1] * 20, list(range(100, 300, 10)), [0] * 20, [777], heads=8, kv_heads=2, dim=128, page=64, seed=11)
    w.build()
    a, la = w.run()
    for _ in range(5):
        b, lb = w.run()
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_strided_query_and_output(salt_lib, ctx):
    w = World(salt_lib, ctx, [2, 1], [50, 7], heads=4, kv_heads=2, dim=64, seed=12)
    w.build()
    a, _ = w.run()
    qkv = torch.full((3, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    qkv[:, 2:6] = w.q.cuda()
    out = torch.full((3, 7, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_attn_run(w.plan, 0, qkv[:, 2:6], out[:, 1:5], w.scale)
    assert torch.equal(out[:, 1:5].cpu(), a) and bool((out[:, [0, 5, 6]] == 7).all())


def test_long_contexts(salt_lib, ctx):
    """70,001 tokens, checked on four of the rows' heads."""
    n, page, dim = 70001, 128, 128
    pages = -(-n // page) + 1
    g = torch.Generator(device="cuda").manual_seed(3)
    c = {m: torch.randn((1, pages, 1, page, dim), generator=g, device="cuda").mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn) for m in "kv"}
    e = {m: torch.randint(118, 122, (1, pages, 1, page), generator=g, device="cuda").to(torch.uint8) for m in "kv"}
    kv = salt_lib.salt_kv_create(ctx, c["k"], c["v"], e["k"], e["v"])
    plan = salt_lib.salt_attn_create(kv, 4, 2, 3, 2 * pages)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).tolist()
    b = dict(q_len=[1, 1], kv_len=[n, 1], page_ptr=[0, pages, pages + 1], pages=order + [order[0]], group=[-1, -1], group_len=[],
             group_page_ptr=[0], group_pages=[])
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch(*b.values()))
    q = torch.randn((2, 4, dim), generator=torch.Generator().manual_seed(1)).bfloat16()
    out, lse = torch.empty((2, 4, dim), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 4), device="cuda")
    salt_lib.salt_attn_run(plan, 0, q.cuda(), out, dim ** -0.5, lse)
    ref = attention(q, value(c["k"][0].view(torch.uint8), e["k"][0]), value(c["v"][0].view(torch.uint8), e["v"][0]), b, page, dim ** -0.5)
    compare(out.cpu(), lse.cpu(), *ref)


def test_offsets_past_32_bits(salt_lib, ctx):
    """A cache of 5 GiB a side, the batch's pages at its end and past 2^32 bytes."""
    heads, page, dim = 8, 128, 128
    pages = (5 << 30) // (heads * page * dim)
    k, v = (torch.empty((1, pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    ke, ve = (torch.empty((1, pages, heads, page), dtype=torch.uint8, device="cuda") for _ in range(2))
    kv = salt_lib.salt_kv_create(ctx, k, v, ke, ve)
    lists = [pages - 1, (1 << 32) // (heads * page * dim) + 1, 3]
    n = 300
    x, y = (torch.randn((n, heads, dim), generator=torch.Generator().manual_seed(i)).bfloat16() for i in (1, 2))
    slots = torch.tensor([lists[j // page] * page + j % page for j in range(n)], dtype=torch.int32, device="cuda")
    salt_lib.salt_kv_write(kv, 0, x.cuda(), y.cuda(), slots)
    plan = salt_lib.salt_attn_create(kv, 8, 1, 2, 3)
    b = dict(q_len=[2], kv_len=[n], page_ptr=[0, 3], pages=[0, 1, 2], group=[-1], group_len=[], group_page_ptr=[0], group_pages=[])
    host = dict(b, pages=lists)
    salt_lib.salt_attn_build(plan, salt_lib.salt_attn_batch(*host.values()))
    q = torch.randn((2, 8, dim), generator=torch.Generator().manual_seed(3)).bfloat16()
    out, lse = torch.empty((2, 8, dim), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 8), device="cuda")
    salt_lib.salt_attn_run(plan, 0, q.cuda(), out, dim ** -0.5, lse)
    at = torch.tensor(lists)
    ref = attention(q, value(k[0, at], ke[0, at]), value(v[0, at], ve[0, at]), b, page, dim ** -0.5)
    compare(out.cpu(), lse.cpu(), *ref)


def test_write_then_attend_on_other_streams(salt_lib, ctx):
    """A plan built on one stream, run on two others and built again: each
    call waits for what it depends on."""
    w = World(salt_lib, ctx, [1] * 8, [400] * 8, [0] * 8, [500], heads=8, kv_heads=2, dim=128, page=64, seed=13)
    out = w.reference()
    s = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(3):
        w.build(s[0])
        res = []
        for st in (s[1], s[2], s[1]):
            with torch.cuda.stream(st):
                o, lse = torch.empty_like(w.q, device="cuda"), torch.empty((w.T, w.heads), device="cuda")
                q = w.q.cuda()
            salt_lib.salt_attn_run(w.plan, 0, q, o, w.scale, lse, st)
            res.append((o, lse))
        torch.cuda.synchronize()
        for o, lse in res:
            compare(o.cpu(), lse.cpu(), *out)


def test_captured_run_follows_the_plan(salt_lib, ctx):
    """A captured run replayed after the plan was built for another batch; a
    larger batch than the capture's is refused."""
    w = World(salt_lib, ctx, [1, 3, 2], [200, 30, 90], [0, -1, 0], [140], heads=8, kv_heads=2, dim=64, page=32, seed=14)
    w.build()
    out, lse = torch.full((8, 8, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((8, 8), 7.0, device="cuda")
    q = torch.zeros((8, 8, 64), dtype=torch.bfloat16, device="cuda")
    q[:6] = w.q.cuda()
    st = torch.cuda.Stream()
    w.build(st)
    salt_lib.salt_attn_run(w.plan, 0, q, out, w.scale, lse, st)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        salt_lib.salt_attn_run(w.plan, 0, q, out, w.scale, lse, st)
    with pytest.raises(salt_lib.SaltError):
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=st):
            w.build(st)
    torch.cuda.synchronize()
    w.build(st)
    with torch.cuda.stream(st):
        graph.replay()
    torch.cuda.synchronize()
    compare(out[:6].cpu(), lse[:6].cpu(), *w.reference())
    old = dict(w.batch)
    w.batch.update(q_len=[2, 1, 0], kv_len=[180, 29, 4])
    out.fill_(7.0)
    with torch.cuda.stream(st):
        out.fill_(7.0)
        w.build(st)
        graph.replay()
    torch.cuda.synchronize()
    w.T = 3
    compare(out[:3].cpu(), lse[:3].cpu(), *attention(q[:3].cpu(), *(value(w.codes[n][0], w.exps[n][0]) for n in "kv"), w.batch, 32, w.scale))
    assert bool((out[3:] == 7).all())
    w.batch = old
    big = World(salt_lib, ctx, [1, 3, 4], [200, 30, 90], heads=8, kv_heads=2, dim=64, page=32, seed=15)
    del big
    plan = salt_lib.salt_attn_create(w.kv, 8, 3, 8, 40, 1)
    w.plan, w.T = plan, 6
    w.build(st)
    torch.cuda.synchronize()
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2, stream=st):
        salt_lib.salt_attn_run(plan, 0, q, out, w.scale, lse, st)
    w.batch.update(q_len=[1, 3, 4])
    with torch.cuda.stream(st):
        out.fill_(7.0)
        w.build(st)
        graph2.replay()
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    assert salt_lib.salt_get_device_error(ctx) == 0x80


def test_refusals(salt_lib, ctx):
    salt = salt_lib
    w = World(salt, ctx, [1, 2], [40, 20], [0, -1], [30], heads=4, kv_heads=2, dim=64, page=16, seed=16)
    out = torch.empty((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    q = w.q.cuda()
    with pytest.raises(salt.SaltError) as e:
        salt.salt_attn_run(w.plan, 0, q, out, 0.1)
    assert e.value.name == "SALT_ERR_NOT_BUILT"
    good = dict(w.batch)
    for change, name in [
            (dict(q_len=[-1, 2]), "SALT_ERR_INVALID_ARG"),
            (dict(q_len=[2, 2]), "SALT_ERR_TOO_MANY_TOKENS"),
            (dict(kv_len=[49, 20]), "SALT_ERR_INVALID_ARG"),      # four pages' tokens, three pages
            (dict(kv_len=[-1, 20]), "SALT_ERR_INVALID_ARG"),
            (dict(kv_len=[2 ** 31 - 1, 20]), "SALT_ERR_INVALID_ARG"),
            (dict(group=[1, -1]), "SALT_ERR_DOMAIN_RANGE"),
            (dict(group=[-2, -1]), "SALT_ERR_DOMAIN_RANGE"),
            (dict(pages=[10 ** 6] + good["pages"][1:]), "SALT_ERR_SLOT_RANGE"),
            (dict(pages=[-1] + good["pages"][1:]), "SALT_ERR_SLOT_RANGE"),
            (dict(group_pages=[10 ** 6, 0]), "SALT_ERR_SLOT_RANGE"),
            (dict(page_ptr=[0, 6, 5]), "SALT_ERR_INVALID_ARG"),
            (dict(page_ptr=[1, 3, 5]), "SALT_ERR_INVALID_ARG")]:
        w.batch = dict(good, **change)
        with pytest.raises((salt.SaltError, ValueError)) as e:
            w.build()
        if isinstance(e.value, salt.SaltError):
            assert e.value.name == name, change
        with pytest.raises(salt.SaltError) as e:  # a failed build leaves no plan
            salt.salt_attn_run(w.plan, 0, q, out, 0.1)
        assert e.value.name == "SALT_ERR_NOT_BUILT"
    w.batch = good
    w.build()
    for layer in (-1, 1):
        with pytest.raises(salt.SaltError) as e:
            salt.salt_attn_run(w.plan, layer, q, out, 0.1)
        assert e.value.name == "SALT_ERR_LAYER_RANGE"
    for scale in (float("nan"), float("inf")):
        with pytest.raises(salt.SaltError) as e:
            salt.salt_attn_run(w.plan, 0, q, out, scale)
        assert e.value.name == "SALT_ERR_INVALID_ARG"
    odd = torch.as_strided(torch.zeros(3 * 260, dtype=torch.bfloat16, device="cuda"), (3, 4, 64), (260, 64, 1))
    for a, b in ((odd, out), (q, odd)):
        with pytest.raises(salt.SaltError) as e:
            salt.salt_attn_run(w.plan, 0, a, b, 0.1)
        assert e.value.name == "SALT_ERR_ALIGN"
    with pytest.raises(ValueError):
        salt.salt_attn_run(w.plan, 0, q[:2], out, 0.1)
    with pytest.raises(ValueError):
        salt.salt_attn_run(w.plan, 0, q, out, 0.1, lse=torch.empty((2, 4), device="cuda"))
    for kw in (dict(n_heads=3), dict(n_heads=0), dict(n_heads=130), dict(max_seqs=0), dict(max_pages=0), dict(max_groups=-1),
               dict(max_tokens=0), dict(max_tokens=16385)):
        args = dict(n_heads=4, max_seqs=2, max_tokens=3, max_pages=9, max_groups=1)
        args.update(kw)
        with pytest.raises(salt.SaltError):
            salt.salt_attn_create(w.kv, **args)
    salt.salt_attn_run(w.plan, 0, q, out, w.scale)
    out_ref = w.reference()[0]
    torch.cuda.synchronize()
    assert float((out.cpu().double() - out_ref).abs().max()) < 0.05
