"""A cached value that stands for NaN spoils every row that sees it, whatever its
probability, and no other row; the log-sums are those of the scores."""
import math

import pytest
import torch

from attn_world import Shared, bf16_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


# requests, query tokens each, query heads (of 8 key/value heads): few items of one tile each, whole items of
# few and of many rows
@pytest.mark.parametrize("kind", [(1, 2, 16), (80, 1, 16), (64, 32, 32)], ids=["split", "narrow", "wide"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("below", [0, 20, 90, 105, 120, 160, 400])
def test_nan_value_of_small_probability(salt_lib, ctx, kind, dim, below):
    """The NaN value's score is `below` binades under the others' (e4m3: to the nearest of 16 a binade)."""
    requests, q, heads = kind
    n, at = 400, 172
    k, v = bf16_rows(n, 8, dim, 1), bf16_rows(n, 8, dim, 2)
    k[..., 0] = 0
    k[at, :, 0] = -below
    v[at] = float("nan")
    # requests of an even number see it, the others end before it
    w = Shared(salt_lib, ctx, k, v, [q] * requests, [n if b % 2 == 0 else at for b in range(requests)], heads)
    w.build()
    w.q[..., 0] = math.log(2) / w.scale
    out, lse = w.run()
    _, ref, _, ltol = w.reference()
    assert bool(((lse.double() - ref).abs() <= ltol).all())
    sees = (torch.arange(w.T, device="cuda") // q) % 2 == 0
    assert bool(torch.isnan(out[sees]).all()) and not bool(torch.isnan(out[~sees]).any())


def test_nan_value_behind_some_rows(salt_lib, ctx):
    """The last token's value: of a chunk's query rows only the last sees it."""
    n, dim = 300, 128
    k, v = bf16_rows(n, 8, dim, 3), bf16_rows(n, 8, dim, 4)
    k[..., 0] = 0
    k[n - 1, :, 0] = -150
    v[n - 1] = float("inf")
    w = Shared(salt_lib, ctx, k, v, [32] * 64, [n] * 64, 32)
    w.build()
    w.q[..., 0] = math.log(2) / w.scale
    out, _ = w.run()
    last = torch.arange(w.T, device="cuda") % 32 == 31
    assert bool(torch.isnan(out[last]).all()) and bool(torch.isfinite(out[~last]).all())
