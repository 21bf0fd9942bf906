"""Scores up to the largest that are served, 2^23 in magnitude: a row is the mean of the
values whose score is the largest, and its log-sum that score (and the logarithm
of their number)."""
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
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("log2", [12, 20, 24, 26])
@pytest.mark.parametrize("best", [(5,), (300,), (7, 9), (100, 390)])
def test_largest_score_takes_all(salt_lib, ctx, kind, sign, log2, best):
    """Keys of one element 2^a, a query of one element: the scores are scale * (+-2^log2) at the best tokens
    and differ from it by half of it at least elsewhere, by powers of two.  2^26 / 8 = 2^23 is the limit."""
    requests, q, heads = kind
    n, dim = 400, 64
    half = log2 // 2
    a = torch.tensor([half - sign * (1 + j % min(7, half)) for j in range(n)], dtype=torch.float64)
    a[list(best)] = half
    k = torch.zeros((n, 8, dim), dtype=torch.bfloat16)
    k[..., 0] = torch.exp2(a)[:, None].bfloat16()
    v = bf16_rows(n, 8, dim, 1)
    v[::3] = (v[::3].double() * 2.0 ** -30).bfloat16()
    w = Shared(salt_lib, ctx, k, v, [q] * requests, [n] * requests, heads)
    w.build()
    w.q.zero_()
    w.q[..., 0] = sign * 2.0 ** (log2 - half)
    out, lse = w.run()
    seen = torch.ones((w.T, len(best)), dtype=torch.bool)
    for i, b in enumerate(best):   # the last rows of a chunk see all tokens, the first ones not the last
        seen[:, i] = b <= n - q + torch.arange(w.T) % q
    G = heads // 8
    V = w.values["v"][list(best)].repeat_interleave(G, 1)                     # [best, heads, dim]
    count = seen.sum(1).cuda()
    ref = torch.einsum("tb,bhd->thd", seen.double().cuda(), V) / count.clamp(min=1)[:, None, None]
    rows = count > 0                                                          # (else the next best one, not looked at)
    tol = ref.abs() * 2.0 ** -8 + 2.0 ** -11 * torch.einsum("tb,bhd->thd", seen.double().cuda(), V.abs())
    assert bool(((out.double() - ref).abs() <= tol)[rows].all())
    s = sign * 2.0 ** log2 * w.scale
    want = s + torch.log(count.double())[:, None]
    assert bool(((lse.double() - want).abs() <= abs(s) * 2.0 ** -21)[rows].all())
    assert math.isfinite(s) and bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
