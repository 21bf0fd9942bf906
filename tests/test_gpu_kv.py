"""The paged 8-bit cache: codes and exponents bit for bit against the 64-bit
definition, rows read back exactly, slots, strides, edges and refusals."""
import pytest
import torch

from attn_reference import quantise, value

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def make_cache(salt, ctx, layers, pages, heads, page, dim, fill=0x7F):
    """Cache tensors between guard bytes; unwritten memory holds NaN codes."""
    t = {}
    for name, shape in (("k", (layers, pages, heads, page, dim)), ("v", (layers, pages, heads, page, dim)),
                        ("k_exp", (layers, pages, heads, page)), ("v_exp", (layers, pages, heads, page))):
        n = 1
        for s in shape:
            n *= s
        buf = torch.full((n + 512,), fill, dtype=torch.uint8, device="cuda")
        t[name] = buf[256:256 + n].view(shape)
        t[name + "_buf"] = buf
    t["kv"] = salt.salt_kv_create(ctx, t["k"], t["v"], t["k_exp"], t["v_exp"])
    return t


def guards_ok(t, fill=0x7F):
    return all(bool((t[n + "_buf"][:256] == fill).all()) and bool((t[n + "_buf"][-256:] == fill).all())
               for n in ("k", "v", "k_exp", "v_exp"))


def rows(n, heads, dim, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, dim), generator=g) * torch.exp(3 * torch.randn((n, heads, 1), generator=g))
    return x.bfloat16()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n,heads", [(1, 1), (1, 8), (3, 5), (130, 2), (777, 3)])
def test_write_and_read_back(salt_lib, ctx, dim, page, n, heads):
    pages = -(-n // page) + 2
    t = make_cache(salt_lib, ctx, 2, pages, heads, page, dim)
    g = torch.Generator().manual_seed(n)
    slots = torch.randperm(pages * page, generator=g)[:n].int()
    slots[n // 2] = -1 if n > 1 else slots[0]
    k, v = rows(n, heads, dim, 1), rows(n, heads, dim, 2)
    salt_lib.salt_kv_write(t["kv"], 1, k.cuda(), v.cuda(), slots.cuda())
    torch.cuda.synchronize()
    assert guards_ok(t) and salt_lib.salt_get_device_error(ctx) == 0
    assert bool((t["k"][0] == 0x7F).all()) and bool((t["v_exp"][0] == 0x7F).all())  # the other layer
    live = slots >= 0
    p, o = slots[live].long() // page, slots[live].long() % page
    untouched = torch.ones((pages, page), dtype=torch.bool)
    untouched[p, o] = False
    for name, x in (("k", k), ("v", v)):
        c, e = quantise(x[live])
        got_c = t[name][1].cpu()[p, :, o].view(torch.float8_e4m3fn).double()
        got_e = t[name + "_exp"][1].cpu()[p, :, o].long()
        assert torch.equal(got_e, e) and torch.equal(got_c, c)
        assert bool((t[name][1].cpu().transpose(1, 2)[untouched] == 0x7F).all())
        assert bool((t[name + "_exp"][1].cpu().transpose(1, 2)[untouched] == 0x7F).all())
    rk, rv = torch.full((n, heads, dim), 7.0).bfloat16().cuda(), torch.full((n, heads, dim), 7.0).bfloat16().cuda()
    salt_lib.salt_kv_read(t["kv"], 1, slots.cuda(), rk, rv)
    for name, got in (("k", rk), ("v", rv)):
        want = value(t[name][1].cpu()[p, :, o], t[name + "_exp"][1].cpu()[p, :, o])
        assert torch.equal(got.cpu()[live].double(), want)  # 4 significant bits: exact in bf16
        assert bool((got.cpu()[~live] == 0).all())


def test_edges_of_the_range(salt_lib, ctx):
    """Zeros, the exact power-of-two boundary, subnormals, the largest finite
    values, infinities and NaN."""
    D = 64
    x = torch.zeros((12, 1, D))
    x[1, 0, 3] = 448.0
    x[2, 0, 3] = 450.0
    x[3, 0, 5] = 1e-40
    x[4, 0] = torch.linspace(-1e-38, 1e-38, D)
    x[5, 0, 0], x[5, 0, 1] = 3.3e38, 1.0
    x[6, 0, 9] = float("inf")
    x[7, 0, 9] = float("nan")
    x[8, 0, :] = -0.0
    x[9, 0, 0], x[9, 0, 1] = 1.0, 2.0 ** -20
    x[10, 0, 0], x[10, 0, 1:] = 448.0, torch.linspace(0, 0.02, D - 1)  # codes down among e4m3's subnormals
    x[11, 0, :] = float("-inf")
    x = x.bfloat16()
    t = make_cache(salt_lib, ctx, 1, 1, 1, 16, D)
    slots = torch.arange(12, dtype=torch.int32).cuda()
    salt_lib.salt_kv_write(t["kv"], 0, x.cuda(), x.cuda(), slots)
    c, e = quantise(x)
    assert torch.equal(t["k_exp"][0, 0, 0, :12].cpu().long(), e[:, 0])
    assert torch.equal(t["k"][0, 0, 0, :12].cpu().view(torch.float8_e4m3fn).double(), c[:, 0])
    assert torch.equal(t["k"].cpu()[0, 0, 0, :12], t["v"].cpu()[0, 0, 0, :12])
    a, b = torch.empty((12, 1, D), dtype=torch.bfloat16, device="cuda"), torch.empty((12, 1, D), dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_kv_read(t["kv"], 0, slots, a, b)
    want = value(t["k"][0, 0, 0, :12], t["k_exp"][0, 0, 0, :12]).float().bfloat16()
    got = a.cpu()[:, 0]
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan) and bool(nan[6].all()) and bool(nan[7].all()) and bool(nan[11].all())
    assert torch.equal(got[~nan], want[~nan])


def test_strided_rows_and_guarded_results(salt_lib, ctx):
    n, heads, dim = 37, 2, 128
    t = make_cache(salt_lib, ctx, 1, 3, heads, 32, dim)
    qkv = rows(n, 8, dim, 3).cuda()  # k: heads 4..5, v: heads 6..7 of fused rows
    slots = torch.randperm(96, generator=torch.Generator().manual_seed(1))[:n].int().cuda()
    salt_lib.salt_kv_write(t["kv"], 0, qkv[:, 4:6], qkv[:, 6:], slots)
    p, o = slots.cpu().long() // 32, slots.cpu().long() % 32
    for name, x in (("k", qkv[:, 4:6]), ("v", qkv[:, 6:])):
        c, e = quantise(x.cpu())
        assert torch.equal(t[name][0].cpu()[p, :, o].view(torch.float8_e4m3fn).double(), c)
    wide = torch.full((n, 8, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_kv_read(t["kv"], 0, slots, wide[:, 1:3], wide[:, 5:7])
    assert bool((wide[:, [0, 3, 4, 7]] == 7.0).all())
    want = value(t["v"][0].cpu()[p, :, o], t["v_exp"][0].cpu()[p, :, o])
    assert torch.equal(wide[:, 5:7].cpu().double(), want)


def test_offsets_past_32_bits(salt_lib, ctx):
    """Pages whose bytes lie past 2^32 of a cache of 5 GiB a side."""
    heads, page, dim = 8, 128, 128
    pages = (5 << 30) // (heads * page * dim)
    k, v = (torch.empty((1, pages, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    ke, ve = (torch.empty((1, pages, heads, page), dtype=torch.uint8, device="cuda") for _ in range(2))
    kv = salt_lib.salt_kv_create(ctx, k, v, ke, ve)
    slots = torch.tensor([pages * page - 1, (pages - 1) * page, (1 << 32) // (heads * dim) + 5, 0], dtype=torch.int32)
    x = rows(4, heads, dim, 5)
    salt_lib.salt_kv_write(kv, 0, x.cuda(), x.cuda(), slots.cuda())
    a, b = (torch.empty((4, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    salt_lib.salt_kv_read(kv, 0, slots.cuda(), a, b)
    c, e = quantise(x)
    want = c * torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - 127).double())[..., None]
    assert torch.equal(a.cpu().double(), want) and torch.equal(b.cpu().double(), want)
    last = slots.long()
    assert torch.equal(k[0, last // page, :, last % page].cpu().view(torch.float8_e4m3fn).double(), c)


def test_bad_slots_are_flagged_and_skipped(salt_lib, ctx):
    t = make_cache(salt_lib, ctx, 1, 2, 1, 16, 64)
    x = rows(4, 1, 64, 6).cuda()
    slots = torch.tensor([32, -2, 5, -1], dtype=torch.int32, device="cuda")
    salt_lib.salt_kv_write(t["kv"], 0, x, x, slots)
    assert salt_lib.salt_get_device_error(ctx) == 0x100
    assert guards_ok(t) and int((t["k_exp"] != 0x7F).sum()) == 1
    out = torch.full((4, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    salt_lib.salt_kv_read(t["kv"], 0, slots, out, out.clone())
    assert salt_lib.salt_get_device_error(ctx) == 0x100
    assert bool((out[[0, 1, 3]] == 0).all()) and not bool((out[2] == 0).all())


def test_refusals(salt_lib, ctx):
    salt = salt_lib
    t = make_cache(salt, ctx, 1, 2, 2, 16, 64)
    x, s = rows(3, 2, 64, 7).cuda(), torch.arange(3, dtype=torch.int32, device="cuda")
    for layer in (-1, 1):
        with pytest.raises(salt.SaltError) as e:
            salt.salt_kv_write(t["kv"], layer, x, x, s)
        assert e.value.name == "SALT_ERR_LAYER_RANGE"
    odd = torch.as_strided(torch.zeros(3 * 132, dtype=torch.bfloat16, device="cuda"), (3, 2, 64), (132, 64, 1))
    with pytest.raises(salt.SaltError) as e:
        salt.salt_kv_write(t["kv"], 0, odd, x, s)
    assert e.value.name == "SALT_ERR_ALIGN"
    with pytest.raises(salt.SaltError) as e:
        salt.salt_kv_read(t["kv"], 0, s, odd, x)
    assert e.value.name == "SALT_ERR_ALIGN"
    with pytest.raises(salt.SaltError) as e:  # rows that overlap
        salt.salt_kv_write(t["kv"], 0, torch.as_strided(x, (3, 2, 64), (64, 64, 1)), x, s)
    assert e.value.name == "SALT_ERR_INVALID_ARG"
    with pytest.raises(ValueError):
        salt.salt_kv_write(t["kv"], 0, x, x, s[:2])
    salt.salt_kv_write(t["kv"], 0, x[:0], x[:0], s[:0])  # no tokens: nothing to do
    for shape, name in (((1, 2, 2, 16, 96), "SALT_ERR_INVALID_ARG"), ((1, 2, 2, 24, 64), "SALT_ERR_INVALID_ARG"),
                        ((1, 2, 2, 256, 64), "SALT_ERR_INVALID_ARG"), ((0, 2, 2, 16, 64), "SALT_ERR_INVALID_ARG")):
        k = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        ex = torch.zeros(shape[:4], dtype=torch.uint8, device="cuda")
        with pytest.raises(salt.SaltError) as e:
            salt.salt_kv_create(ctx, k, k, ex, ex)
        assert e.value.name == name
    with pytest.raises(ValueError):
        salt.salt_kv_create(ctx, t["k"], t["v"], t["k_exp"][0], t["v_exp"])
    assert salt.salt_get_device_error(ctx) == 0
