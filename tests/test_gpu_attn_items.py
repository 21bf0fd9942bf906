"""Items of several tiles and CTAs of several items, by the plan's own account:
stages that are used again, scores that run into the next item, queries in both
buffers, references that move in later tiles, rows of items that are split."""
import numpy as np
import pytest
import torch

from attn_world import Shared, bf16_rows, compare

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def checked(salt, w, **least):
    """Runs and compares; `least`: what the plan has at least."""
    w.build()
    shape = salt.salt_attn_get_shape(w.plan)
    for k, n in least.items():
        assert shape[k] >= n, shape
    got = w.run()
    compare(*got, *w.reference())
    return got, shape


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv_heads, heads, q", [(8, 32, 32), (8, 8, 100), (4, 20, 51), (2, 16, 63), (16, 16, 70)])
def test_wide_items(salt_lib, ctx, kv_heads, heads, q, dim):
    r = np.random.RandomState(heads + q)
    own = r.randint(1, 900, 64).tolist()
    w = Shared(salt_lib, ctx, bf16_rows(1100, kv_heads, dim, 1), bf16_rows(1100, kv_heads, dim, 2), [q - b % 7 for b in range(64)], own,
               heads, prompt=200, page=32)
    _, shape = checked(salt_lib, w, wide_tiles=2)
    assert shape["wide_items"] > shape["wide_ctas"], shape


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kv_heads, heads, q", [(8, 32, 1), (8, 16, 2), (4, 12, 5), (8, 8, 4), (2, 2, 3)])
def test_narrow_items(salt_lib, ctx, kv_heads, heads, q, dim):
    requests = 1400 // kv_heads
    r = np.random.RandomState(heads + q)
    own = r.randint(q, 1000, requests).tolist()
    w = Shared(salt_lib, ctx, bf16_rows(1000, kv_heads, dim, 3), bf16_rows(1000, kv_heads, dim, 4), [q] * requests, own, heads, page=16)
    _, shape = checked(salt_lib, w, narrow_tiles=3)
    assert shape["narrow_items"] > 2 * shape["narrow_ctas"], shape


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_scale", [1.0, 8.0, 40.0])
def test_both_kinds_with_wild_scores(salt_lib, ctx, q_scale, dim):
    """A decode batch behind a prompt beside some chunks; the larger the scores, the more often a
    row's reference moves after its first tile."""
    r = np.random.RandomState(dim)
    q = [1] * 150 + [40, 7, 64] * 8
    own = r.randint(1, 800, len(q)).tolist()
    w = Shared(salt_lib, ctx, bf16_rows(1500, 8, dim, 5, spread=1.0), bf16_rows(1500, 8, dim, 6, spread=1.0), q, own, 32, prompt=700, page=128)
    w.q *= q_scale
    _, shape = checked(salt_lib, w, wide_tiles=2, narrow_tiles=2, combined=1)
    assert shape["narrow_items"] > shape["narrow_ctas"], shape


@pytest.mark.parametrize("kind", [(80, 1, 16), (64, 32, 32)], ids=["narrow", "wide"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("step", [4.0, 10.0, 14.0, 40.0, 100.0])
def test_a_maximum_that_grows(salt_lib, ctx, kind, dim, step):
    """Each tile's largest score is above the last one's by `step`."""
    requests, q, heads = kind
    n = 640
    k, v = bf16_rows(n, 8, dim, 7), bf16_rows(n, 8, dim, 8)
    k[..., 0] = (torch.arange(n) // 128 * step)[:, None]
    w = Shared(salt_lib, ctx, k, v, [q] * requests, [n] * requests, heads)
    w.q[..., 0] = dim ** 0.5
    _, shape = checked(salt_lib, w)
    assert max(shape["wide_tiles"], shape["narrow_tiles"]) == 5, shape


def test_rows_that_see_nothing_in_long_items(salt_lib, ctx):
    """Chunks longer than their cached tokens, beside ordinary ones, without and behind a prompt."""
    for prompt in (0, 300):
        own = [0, 3, 40, 600, 599, 64, 1, 500] * 8
        w = Shared(salt_lib, ctx, bf16_rows(900, 8, 64, 9), bf16_rows(900, 8, 64, 10), [64] * 64, own, 32, prompt=prompt)
        (out, lse), _ = checked(salt_lib, w, wide_tiles=3)
        if prompt == 0:
            assert bool(torch.isinf(lse[:64]).all()) and bool((out[:64] == 0).all())


def test_same_bits_beside_other_work(salt_lib, ctx):
    """Long items repeat bit for bit, also while other kernels take SMs away."""
    r = np.random.RandomState(0)
    q = [1] * 100 + [50] * 20
    w = Shared(salt_lib, ctx, bf16_rows(1200, 8, 128, 11), bf16_rows(1200, 8, 128, 12), q, r.randint(50, 700, len(q)).tolist(), 32, prompt=500)
    (out, lse), _ = checked(salt_lib, w, wide_tiles=2, narrow_tiles=2)
    busy, st = torch.randn((3000, 3000), device="cuda"), torch.cuda.Stream()
    for i in range(8):
        if i % 2:
            with torch.cuda.stream(st):
                busy = busy @ busy * 1e-2
        again = w.run()
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_shape_of_a_plan(salt_lib, ctx):
    w = Shared(salt_lib, ctx, bf16_rows(40, 2, 64, 13), bf16_rows(40, 2, 64, 14), [1, 2], [40, 30], 4)
    before = salt_lib.salt_attn_get_shape(w.plan)
    assert before["wide_items"] == before["narrow_items"] == before["combined"] == 0 and before["workspace_bytes"] >= 2 * 3 * 4 * 65 * 4
    w.build()
    s = salt_lib.salt_attn_get_shape(w.plan)
    assert (s["wide_items"], s["wide_tiles"], s["narrow_items"], s["narrow_tiles"]) == (0, 0, 4, 1)
