"""The softmax's sums where value rows are very small or zero: a row's
reference follows its largest probability times value, its sum the
probabilities alone, and the two may lie 2^100 apart.  Batches of as many
requests as leave items whole, so that an item's reference moves in its later
tiles."""
import math

import pytest
import torch

from attn_world import Shared, bf16_rows, compare

pytestmark = pytest.mark.gpu

# requests, query tokens each, query heads (of 8 key/value heads): rows of few query tokens and of many
NARROW, WIDE = (80, 1, 16), (64, 32, 32)


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def world(salt, ctx, kind, k, v, **kw):
    requests, q, heads = kind
    w = Shared(salt, ctx, k, v, [q] * requests, [len(k)] * requests, heads, **kw)
    w.build()
    return w


@pytest.mark.parametrize("kind", [NARROW, WIDE], ids=["narrow", "wide"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("leading", [1, 128, 256, 300])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -40, 2.0 ** -110])
def test_small_values_before_ordinary_ones(salt_lib, ctx, kind, dim, leading, small):
    """Leading tokens of zero or tiny values keep their share of the probability."""
    n = 500
    k, v = bf16_rows(n, 8, dim, 1), bf16_rows(n, 8, dim, 2)
    v[:leading] = (v[:leading].double() * small).bfloat16()
    w = world(salt_lib, ctx, kind, k, v)
    compare(*w.run(), *w.reference())


@pytest.mark.parametrize("kind", [NARROW, WIDE], ids=["narrow", "wide"])
@pytest.mark.parametrize("binades", [0, 10, 30, 50, 100, 126])
@pytest.mark.parametrize("gap", [15.0, 17.0, 100.0, 117.0, 129.0, 150.0, 180.0, 203.0, 300.0])
def test_a_large_score_of_a_small_value(salt_lib, ctx, kind, binades, gap):
    """One late token's score is `gap` binades above all others, its value row
    `binades` below theirs (126: zero)."""
    n, dim = 450, 64
    k, v = bf16_rows(n, 8, dim, 3), bf16_rows(n, 8, dim, 4)
    k[..., 0] = 0
    k[300, :, 0] = gap
    v[300] = (v[300].double() * (0.0 if binades == 126 else 2.0 ** -binades)).bfloat16()
    w = world(salt_lib, ctx, kind, k, v)
    w.q[..., 0] = math.log(2) / w.scale
    compare(*w.run(), *w.reference())


@pytest.mark.parametrize("kind", [NARROW, WIDE], ids=["narrow", "wide"])
def test_many_large_scores_of_zero_values(salt_lib, ctx, kind):
    """9,000 zero rows 113.6 binades above one ordinary row, in the tiles after its
    own: each one's probability is just below what moves the reference."""
    n, dim = 9000, 64
    k = torch.zeros((n, 8, dim), dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    k[128:, :, 0] = 112.0
    v[0] = 1.0
    w = world(salt_lib, ctx, kind, k, v, page=128)
    w.q[..., 0] = 5.625                        # 112 * 5.625 / 8 = 113.6 log 2
    compare(*w.run(), *w.reference())


@pytest.mark.parametrize("kind", [NARROW, WIDE], ids=["narrow", "wide"])
def test_a_key_that_is_nan_before_a_large_score(salt_lib, ctx, kind):
    """A row that saw a NaN stays NaN when its reference moves, out and log-sum both."""
    n, dim = 450, 64
    k, v = bf16_rows(n, 8, dim, 5), bf16_rows(n, 8, dim, 6)
    k[..., 0] = 0
    k[172, :, 0] = float("nan")
    k[300, :, 0] = 400.0                       # the same place of its tile
    v[300] = 0
    w = world(salt_lib, ctx, kind, k, v)
    w.q[..., 0] = math.log(2) / w.scale
    out, lse = w.run()
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())
