"""Norms and rotation of heads: against the 64-bit definition, rows and cache,
strides, in place, positions, edges and refusals."""
import math

import pytest
import torch

from attn_reference import quantise
from rope_reference import check_bf16, check_codes, frequencies, rotate
from test_gpu_kv import guards_ok, make_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def heads_of(n, heads, dim, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, heads, dim), generator=g) * torch.exp(torch.randn((n, heads, 1), generator=g))).bfloat16()


def weights_of(dim, seed):
    return (1.0 + 0.3 * torch.randn(dim, generator=torch.Generator().manual_seed(seed))).bfloat16()


def places(n, far, seed):
    return torch.randint(0, far, (n,), generator=torch.Generator().manual_seed(seed)).int()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 0)])
@pytest.mark.parametrize("n,heads,kv_heads,norms", [(1, 8, 2, "qk"), (3, 1, 1, ""), (37, 5, 3, "k"), (200, 3, 2, "q")])
def test_rows(salt_lib, ctx, n, heads, kv_heads, norms, dim, rot, interleaved):
    q, k, pos, freq = heads_of(n, heads, dim, 1), heads_of(n, kv_heads, dim, 2), places(n, 200000, 3), frequencies(rot)
    wq, wk = (weights_of(dim, 4) if "q" in norms else None), (weights_of(dim, 5) if "k" in norms else None)
    rope = salt_lib.salt_rope_create(ctx, dim, rot, freq, interleaved, scale=1.25, eps=1e-5, norm_offset=0.5)
    # rows of a wider buffer, whose other elements stay
    qo = torch.full((n, heads + 1, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    ko = torch.full((n, kv_heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    fused = torch.cat([q, k], 1).cuda()
    salt_lib.salt_rope_apply(rope, fused[:, :heads], fused[:, heads:], pos.cuda(), qo[:, :heads], ko,
                             None if wq is None else wq.cuda(), None if wk is None else wk.cuda())
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0 and bool((qo[:, heads:] == 7.0).all())
    for x, w, got in ((q, wq, qo[:, :heads]), (k, wk, ko)):
        want, tol = rotate(x, pos, freq, interleaved, w, 1e-5, 0.5, 1.25)
        check_bf16(got.cpu(), want, tol)
    # in place
    salt_lib.salt_rope_apply(rope, fused[:, :heads], fused[:, heads:], pos.cuda(), fused[:, :heads], fused[:, heads:],
                             None if wq is None else wq.cuda(), None if wk is None else wk.cuda())
    torch.cuda.synchronize()
    assert torch.equal(fused[:, :heads], qo[:, :heads]) and torch.equal(fused[:, heads:], ko)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot,page", [(64, 32, 16), (64, 64, 128), (128, 128, 64), (128, 16, 32)])
@pytest.mark.parametrize("n,heads,kv_heads,norm", [(1, 4, 1, True), (5, 3, 3, False), (150, 10, 2, True)])
def test_into_the_cache(salt_lib, ctx, n, heads, kv_heads, norm, dim, rot, page, interleaved):
    pages = -(-n // page) + 2
    t = make_cache(salt_lib, ctx, 2, pages, kv_heads, page, dim)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(n))[:n].int()
    if n > 1:
        slots[n // 2] = -1
    q, k, v, pos, freq = heads_of(n, heads, dim, 1), heads_of(n, kv_heads, dim, 2), heads_of(n, kv_heads, dim, 6), places(n, 10 ** 6, 3), frequencies(rot)
    wq, wk = (weights_of(dim, 4), weights_of(dim, 5)) if norm else (None, None)
    rope = salt_lib.salt_rope_create(ctx, dim, rot, freq, interleaved)
    qkv = torch.cat([q, k, v], 1).cuda()
    qo = torch.full((n, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_rope_write(rope, t["kv"], 1, qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], pos.cuda(),
                             slots.cuda(), qo, *(w if w is None else w.cuda() for w in (wq, wk)))
    torch.cuda.synchronize()
    assert guards_ok(t) and salt_lib.salt_get_device_error(ctx) == 0
    check_bf16(qo.cpu(), *rotate(q, pos, freq, interleaved, wq))
    live = slots >= 0
    p, o = slots[live].long() // page, slots[live].long() % page
    untouched = torch.ones((pages, page), dtype=torch.bool)
    untouched[p, o] = False
    for x in ("k", "v", "k_exp", "v_exp"):
        assert bool((t[x][0] == 0x7F).all()) and bool((t[x][1].cpu().transpose(1, 2)[untouched] == 0x7F).all())
    c, e = quantise(v[live])
    assert torch.equal(t["v"][1].cpu()[p, :, o].view(torch.float8_e4m3fn).double(), c)
    assert torch.equal(t["v_exp"][1].cpu()[p, :, o].long(), e)
    want, tol = rotate(k, pos, freq, interleaved, wk)
    check_codes(t["k"][1].cpu()[p, :, o].view(torch.float8_e4m3fn).double(), t["k_exp"][1].cpu()[p, :, o], want[live], tol[live])


def test_without_norm_and_rotation_it_is_the_plain_write(salt_lib, ctx):
    n, heads, dim, page = 77, 3, 128, 16
    a, b = (make_cache(salt_lib, ctx, 1, 6, heads, page, dim) for _ in range(2))
    k, v = heads_of(n, heads, dim, 1), heads_of(n, heads, dim, 2)
    k[5, 1, 3], v[6, 0, 7], k[7] = math.nan, math.inf, 0.0
    k, v, slots, pos = k.cuda(), v.cuda(), torch.randperm(6 * page)[:n].int().cuda(), torch.arange(n, dtype=torch.int32, device="cuda")
    salt_lib.salt_kv_write(a["kv"], 0, k, v, slots)
    rope = salt_lib.salt_rope_create(ctx, dim, 0, [])
    none = torch.empty((n, 0, dim), dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_rope_write(rope, b["kv"], 0, none, k, v, pos, slots, none)
    torch.cuda.synchronize()
    for x in ("k", "v", "k_exp", "v_exp"):
        assert torch.equal(a[x], b[x])
    assert guards_ok(b)


def test_positions_of_the_whole_range(salt_lib, ctx):
    """Angles keep their digits at the ends of int32, where a product in 64 bits has lost some."""
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 12345, -77777777, 16777217], dtype=torch.int32)
    dim = 128
    freq = frequencies(dim)
    freq[0], freq[1], freq[2] = 2 * math.pi, -1.0, 0.0
    x = heads_of(len(pos), 2, dim, 1)
    rope = salt_lib.salt_rope_create(ctx, dim, dim, freq)
    y, none = torch.empty_like(x).cuda(), torch.empty((len(pos), 0, dim), dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_rope_apply(rope, x.cuda(), none, pos.cuda(), y, none)
    torch.cuda.synchronize()
    check_bf16(y.cpu(), *rotate(x, pos, freq))


@pytest.mark.parametrize("dim", [64, 128])
def test_edges_of_the_range(salt_lib, ctx, dim):
    """Rows of zeros, of elements whose squares leave fp32's range or vanish in it, infinities and NaN: each
    spoils its own head alone."""
    x = heads_of(8, 3, dim, 1)
    x[0] = 0.0
    x[1, 0] *= 2.0 ** 100
    x[1, 1] = 3e38
    x[1, 2] *= 2.0 ** -100
    x[2, 1, 5], x[3, 0, 1], x[4, 2, 0] = math.inf, -math.inf, math.nan
    pos, freq, w = places(8, 5000, 2), frequencies(dim), weights_of(dim, 3)
    t = make_cache(salt_lib, ctx, 1, 1, 3, 16, dim)
    slots = torch.arange(8, dtype=torch.int32, device="cuda")
    rope = salt_lib.salt_rope_create(ctx, dim, dim, freq)
    for norm in (None, w):
        y = torch.empty_like(x).cuda()
        g = None if norm is None else norm.cuda()
        salt_lib.salt_rope_write(rope, t["kv"], 0, x.cuda(), x.cuda(), x.cuda(), pos.cuda(), slots, y, g, g)
        torch.cuda.synchronize()
        fine = torch.isfinite(x).all(-1)
        want, tol = rotate(x, pos, freq, False, norm)
        got, e = y.cpu(), t["k_exp"][0, 0].T[:8].cpu()
        if norm is None:  # 3e38 (cos - sin) may pass the range, in fp32 or on the way to bf16
            big = want.abs().amax(-1) >= 3.3e38
            assert bool((e[fine & ~big] < 255).all()) and bool(big[1, 1])
            fine = fine & ~big
        check_bf16(got[fine], want[fine], tol[fine])
        codes = t["k"][0, 0].transpose(0, 1)[:8].cpu().view(torch.float8_e4m3fn).double()
        check_codes(codes[fine], e[fine], want[fine], tol[fine])
        spoiled = ~torch.isfinite(x).all(-1)
        assert bool((e[spoiled] == 255).all()) and bool((codes[spoiled] == 0).all())
        assert bool((~torch.isfinite(got.float())).any(-1)[spoiled].all())
    assert salt_lib.salt_get_device_error(ctx) == 0 and guards_ok(t)


def test_slots_outside_the_cache(salt_lib, ctx):
    t = make_cache(salt_lib, ctx, 1, 2, 1, 16, 64)
    x = heads_of(4, 1, 64, 1).cuda()
    slots, pos = torch.tensor([32, -2, 3, -1], dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    y = torch.zeros_like(x)
    rope = salt_lib.salt_rope_create(ctx, 64, 64, frequencies(64))
    salt_lib.salt_rope_write(rope, t["kv"], 0, x, x, x, pos, slots, y)
    assert salt_lib.salt_get_device_error(ctx) == 0x100
    assert torch.equal(y, x) and guards_ok(t)   # (position 0)
    written = (t["k"][0, :, 0] != 0x7F).any(-1).flatten().cpu()
    assert written.nonzero().flatten().tolist() == [3]


def test_many_tokens_and_heads(salt_lib, ctx):
    """Several launches' worth of rows a token, and more tokens than fill the SMs at a row a warp."""
    n, heads, dim = 3, 20000, 64
    x, pos, freq = heads_of(n, heads, dim, 1), places(n, 9999, 2), frequencies(dim)
    rope = salt_lib.salt_rope_create(ctx, dim, dim, freq)
    y, none = torch.empty_like(x).cuda(), torch.empty((n, 0, dim), dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_rope_apply(rope, x.cuda(), none, pos.cuda(), y, none)
    check_bf16(y.cpu(), *rotate(x, pos, freq))
    n, heads = 20000, 3
    x, pos = heads_of(n, heads, dim, 3).cuda(), places(n, 50, 4).cuda()
    y, none = torch.empty_like(x), torch.empty((n, 0, dim), dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_rope_apply(rope, none, x, pos, none, y)
    table = torch.stack([rotate(torch.ones((1, 1, dim)), [p], freq)[0][0, 0] for p in range(50)]).cuda()  # cos - sin | cos + sin
    cos, sin = (table[:, 32:] + table[:, :32]) / 2, (table[:, 32:] - table[:, :32]) / 2
    c, s, xd = cos[pos.long()][:, None], sin[pos.long()][:, None], x.double()
    want = torch.cat([xd[..., :32] * c - xd[..., 32:] * s, xd[..., 32:] * c + xd[..., :32] * s], -1)
    tol = (xd[..., :32].abs() + xd[..., 32:].abs()).repeat(1, 1, 2) * 2.0 ** -20
    check_bf16(y, want, tol)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 17, 4), (128, 4, 1), (64, 33, 3), (64, 40, 8)])
def test_warps_that_take_many_rows(salt_lib, ctx, dim, heads, kv_heads, interleaved):
    """Tokens enough that a warp goes over all rows of one, with an odd or even number of passes: rows as in calls of a few tokens, where each pass
    has a warp; into the cache, and in place."""
    n, few, page = 5001, 120, 64
    q, k, v, pos, freq = heads_of(n, heads, dim, 1), heads_of(n, kv_heads, dim, 2), heads_of(n, kv_heads, dim, 3), places(n, 10 ** 6, 4), frequencies(dim)
    wq, wk = weights_of(dim, 5).cuda(), weights_of(dim, 6).cuda()
    rope = salt_lib.salt_rope_create(ctx, dim, dim, freq, interleaved)
    a, b = (make_cache(salt_lib, ctx, 1, n // page + 2, kv_heads, page, dim) for _ in range(2))
    qkv, at = torch.cat([q, k, v], 1).cuda(), pos.cuda()
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(7)).int().cuda()
    split = lambda x: (x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:])  # noqa: E731
    q1, q2, k2 = torch.zeros((n, heads, dim), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, heads, dim), dtype=torch.bfloat16, device="cuda"), k.cuda()
    salt_lib.salt_rope_write(rope, a["kv"], 0, *split(qkv), at, slots, q1, wq, wk)
    for i in range(0, n, few):
        part = slice(i, i + few)
        salt_lib.salt_rope_write(rope, b["kv"], 0, *split(qkv[part]), at[part], slots[part], q2[part], wq, wk)
        salt_lib.salt_rope_apply(rope, qkv[part, :0], k2[part], at[part], qkv[part, :0], k2[part], wq, wk)
    salt_lib.salt_rope_apply(rope, *split(qkv)[:2], at, *split(qkv)[:2], wq, wk)
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0 and guards_ok(a) and guards_ok(b)
    assert torch.equal(q1, q2) and all(torch.equal(a[x], b[x]) for x in ("k", "v", "k_exp", "v_exp"))
    assert torch.equal(qkv[:, :heads], q1) and torch.equal(qkv[:, heads:heads + kv_heads], k2) and torch.equal(qkv[:, heads + kv_heads:].cpu(), v)
    some = torch.arange(0, n, 97)
    check_bf16(q1.cpu()[some], *rotate(q[some], pos[some], freq, interleaved, wq.cpu()))
    check_bf16(k2.cpu()[some], *rotate(k[some], pos[some], freq, interleaved, wk.cpu()))


def test_captured_and_on_another_stream(salt_lib, ctx):
    n, dim = 40, 128
    x, pos, freq = heads_of(n, 4, dim, 1).cuda(), places(n, 1000, 2).cuda(), frequencies(dim)
    rope = salt_lib.salt_rope_create(ctx, dim, dim, freq)
    y, none = torch.zeros_like(x), torch.empty((n, 0, dim), dtype=torch.bfloat16, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        salt_lib.salt_rope_apply(rope, x, none, pos, y, none)
    x.copy_(heads_of(n, 4, dim, 7))
    graph.replay()
    z = torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    salt_lib.salt_rope_apply(rope, x, none, pos, z, none, stream=side)
    torch.cuda.synchronize()
    check_bf16(y.cpu(), *rotate(x.cpu(), pos.cpu(), freq))
    assert torch.equal(y, z)


def test_refusals(salt_lib, ctx):
    f = frequencies(64)

    def refused(name, call):
        with pytest.raises(salt_lib.SaltError) as e:
            call()
        assert e.value.name == name, e.value

    bad = "SALT_ERR_INVALID_ARG"
    for kw in (dict(head_dim=96, rot_dim=64), dict(head_dim=64, rot_dim=128, inv_freq=frequencies(128)), dict(rot_dim=24, inv_freq=f[:12]),
               dict(rot_dim=-16, inv_freq=[]), dict(scale=math.inf), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=1e-40),
               dict(norm_offset=math.nan), dict(inv_freq=[7.0] + f[1:]), dict(inv_freq=[math.nan] + f[1:])):
        refused(bad, lambda: salt_lib.salt_rope_create(ctx, **{**dict(head_dim=64, rot_dim=64, inv_freq=f), **kw}))
    rope = salt_lib.salt_rope_create(ctx, 64, 64, f)
    t, wide = make_cache(salt_lib, ctx, 1, 2, 2, 16, 64), make_cache(salt_lib, ctx, 1, 2, 2, 16, 128)
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    odd = torch.zeros(4 * 2 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(4, 2, 64)
    apart = torch.zeros((4, 2 * 64 + 4), dtype=torch.bfloat16, device="cuda")[:, :128].unflatten(1, (2, 64))
    w = torch.zeros(72, dtype=torch.bfloat16, device="cuda")
    refused("SALT_ERR_ALIGN", lambda: salt_lib.salt_rope_apply(rope, odd, x, i, x, x))
    refused("SALT_ERR_ALIGN", lambda: salt_lib.salt_rope_apply(rope, x, apart, i, x, x))
    refused("SALT_ERR_ALIGN", lambda: salt_lib.salt_rope_apply(rope, x, x, i, x, x, w[4:68]))
    refused("SALT_ERR_LAYER_RANGE", lambda: salt_lib.salt_rope_write(rope, t["kv"], 1, x, x, x, i, i, x))
    refused(bad, lambda: salt_lib.salt_rope_write(rope, wide["kv"], 0, x, x, x, i, i, x))
    lib = salt_lib._lib
    p = x.data_ptr()
    s = torch.cuda.current_stream().cuda_stream
    assert lib.salt_rope_apply(rope.handle, 4, p, 120, 2, p, 128, 2, None, None, i.data_ptr(), p, 128, p, 128, s) == 1
    assert lib.salt_rope_apply(rope.handle, 4, p, 128, 2, None, 128, 2, None, None, i.data_ptr(), p, 128, p, 128, s) == 1
    assert lib.salt_rope_apply(rope.handle, 4, p, 128, 2, p, 128, 2, None, None, None, p, 128, p, 128, s) == 1
    assert lib.salt_rope_apply(rope.handle, -1, p, 128, 2, p, 128, 2, None, None, i.data_ptr(), p, 128, p, 128, s) == 1
    assert lib.salt_rope_apply(rope.handle, 4, p, 128, 0, p, 128, 0, None, None, i.data_ptr(), p, 128, p, 128, s) == 1
    assert lib.salt_rope_write(rope.handle, t["kv"].handle, 0, 4, p, 128, 2, p, 128, p, 128, None, None, i.data_ptr(), None, p, 128, s) == 1
    assert lib.salt_rope_apply(rope.handle, 0, None, 0, 2, None, 0, 2, None, None, None, None, 0, None, 0, s) == 0
    for args in ((x.float(), x, i, x, x), (x, x[:3], i, x, x), (x, x, i[:3], x, x), (x, x, i.long(), x, x), (x, x, i, x[:, :1], x), (x[:, :, ::2], x, i, x, x),
                 (x.cpu(), x, i, x, x)):
        with pytest.raises(ValueError):
            salt_lib.salt_rope_apply(rope, *args)
    with pytest.raises(ValueError):
        salt_lib.salt_rope_create(ctx, 64, 64, f[:5])
    torch.cuda.synchronize()
    assert salt_lib.salt_get_device_error(ctx) == 0 and guards_ok(t) and bool((x == 0).all())
