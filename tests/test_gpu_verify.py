"""Drafted tokens accepted and replaced, number for number against whole-number
arithmetic of Python."""
import numpy as np
import pytest
import torch

from attn_reference import verify

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


def call(salt, ctx, ptr, tok, p, q, u, su, pad=0):
    n, V = len(ptr) - 1, p.shape[1]
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    P = torch.full((p.shape[0], V + pad), float("nan"), device="cuda")
    Q = torch.full((max(len(tok), 1), V + pad), float("nan"), device="cuda")
    P[:, :V] = f(p)
    if len(tok):
        Q[:, :V] = f(q)
    res = torch.full((2, n + 2), 77, dtype=torch.int32, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    salt.salt_verify_drafts(ctx, i32(ptr), i32(tok), P[:, :V], Q[:len(tok), :V], f(np.asarray(u, np.float32)),
                            f(np.asarray(su, np.float32)), res[0, 1:n + 1], res[1, 1:n + 1])
    torch.cuda.synchronize()
    assert bool((res[:, 0] == 77).all()) and bool((res[:, n + 1] == 77).all())
    return res[0, 1:n + 1].tolist(), res[1, 1:n + 1].tolist()


def draws(n, d_hi, V, seed, gap=0.7):
    r = np.random.RandomState(seed)
    d = r.randint(0, d_hi + 1, n)
    ptr = [0] + np.cumsum(d).tolist()
    D = ptr[-1]
    z = 2 * r.randn(D + n, V)
    p = np.exp(z - z.max(1, keepdims=True))
    p = (p / p.sum(1, keepdims=True)).astype(np.float32)
    at = [ptr[b] + b + j for b in range(n) for j in range(d[b])]
    z = z[at] + gap * r.randn(D, V)
    q = np.exp(z - z.max(1, keepdims=True)) if D else np.zeros((0, V))
    q = (q / q.sum(1, keepdims=True)).astype(np.float32) if D else q.astype(np.float32)
    tok = [int(np.argmax(q[i] / r.exponential(size=V))) for i in range(D)]
    return ptr, tok, p, q, r.rand(D).astype(np.float32), r.rand(n).astype(np.float32)


@pytest.mark.parametrize("V", [1, 2, 31, 32, 33, 1000, 1025, 32003, 131072])
@pytest.mark.parametrize("n,d_hi,pad", [(1, 0, 0), (1, 4, 5), (7, 7, 0), (3, 2, 3)])
def test_against_whole_numbers(salt_lib, ctx, V, n, d_hi, pad):
    a = draws(n, d_hi, V, 100 * n + V)
    assert call(salt_lib, ctx, *a, pad=pad) == tuple(verify(*a))
    assert salt_lib.salt_get_device_error(ctx) == 0


def test_many_requests(salt_lib, ctx):
    a = draws(300, 3, 257, 9)
    acc, nxt = call(salt_lib, ctx, *a)
    assert (acc, nxt) == tuple(verify(*a))
    assert len(set(acc)) > 2


def test_more_drafts_than_threads(salt_lib, ctx):
    n, V = 2500, 3
    p, q = np.full((n + 1, V), 1 / 3, np.float32), np.full((n, V), 1 / 3, np.float32)
    u = np.zeros(n, np.float32)
    u[2300] = 1.5
    u[2400] = 1.5
    assert call(salt_lib, ctx, [0, n], [1] * n, p, q, u, [0.5])[0] == [2300]
    assert call(salt_lib, ctx, [0, n], [1] * n, p, q, u * 0, [0.999]) == ([n], [2])


def test_edges_of_the_draw(salt_lib, ctx):
    V = 5000
    one = np.zeros((2, V), np.float32)
    one[0, 17] = 1.0            # accepted, then the last row's draw
    one[1, V - 1] = 1.0
    q = np.zeros((1, V), np.float32)
    q[0, 17] = 1.0
    for su in (0.0, 0.5, np.float32(0.99999994)):
        assert call(salt_lib, ctx, [0, 1], [17], one, q, [0.9], [su]) == ([1], [V - 1])
    # rejected with p equal to q: no residual, p itself is drawn from
    assert call(salt_lib, ctx, [0, 1], [17], one, q, [1.0], [0.3]) == ([0], [17])
    # a row without weight
    assert call(salt_lib, ctx, [0], [], np.zeros((0, V), np.float32), np.zeros((0, V), np.float32), [], []) == ([], [])
    none = np.zeros((1, V), np.float32)
    none[0, 3] = -1.0
    none[0, 4] = np.nan
    assert call(salt_lib, ctx, [0, 0], [], none, np.zeros((0, V), np.float32), [], [0.2]) == ([0], [-1])
    # NaN probabilities of a drafted token reject it; infinite and negative weights count as 1 and 0
    bad = np.zeros((2, V), np.float32)
    bad[0, 9] = np.nan
    bad[0, 11] = np.inf
    bad[0, 12] = -np.inf
    qq = np.zeros((1, V), np.float32)
    assert call(salt_lib, ctx, [0, 1], [9], bad, qq, [0.0], [0.9]) == ([0], [11])
    # two tokens of equal weight: the boundary belongs to the second
    two = np.zeros((1, V), np.float32)
    two[0, 40] = two[0, 4040] = 0.5
    assert call(salt_lib, ctx, [0, 0], [], two, np.zeros((0, V), np.float32), [], [0.5]) == ([0], [4040])
    below = np.nextafter(np.float32(0.5), np.float32(0))
    assert call(salt_lib, ctx, [0, 0], [], two, np.zeros((0, V), np.float32), [], [below]) == ([0], [40])
    assert salt_lib.salt_get_device_error(ctx) == 0


def test_bad_drafts_are_flagged(salt_lib, ctx):
    V = 64
    p, q = np.full((4, V), 1 / V, np.float32), np.full((2, V), 1 / V, np.float32)
    acc, nxt = call(salt_lib, ctx, [0, 1, 2], [V, -1], p, q, [0.0, 0.0], [0.1, 0.1])
    assert acc == [0, 0] and nxt == [6, 6]  # not accepted; p = q, so p is drawn from: the first v with 64 (v + 1) > 640.4
    assert salt_lib.salt_get_device_error(ctx) == 0x200
    acc, nxt = call(salt_lib, ctx, [1, 0, 7], [1, 1], p, q, [0.0, 0.0], [0.1, 0.1])
    assert acc == [0, 0] and nxt == [-1, -1]
    assert salt_lib.salt_get_device_error(ctx) == 0x200


def test_refusals(salt_lib, ctx):
    salt = salt_lib
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    p, q = torch.rand((2, 8), device="cuda"), torch.rand((1, 8), device="cuda")
    u, su = torch.rand(1, device="cuda"), torch.rand(1, device="cuda")
    a, b = i32([0]), i32([0])
    salt.salt_verify_drafts(ctx, i32([0, 1]), i32([3]), p, q, u, su, a, b)
    for kw in (dict(target_p=p[:1]), dict(draft_p=q[:, :7]), dict(accept_u=su.double()), dict(draft_ptr=i32([0]))):
        args = dict(draft_ptr=i32([0, 1]), draft_tokens=i32([3]), target_p=p, draft_p=q, accept_u=u, sample_u=su)
        args.update(kw)
        with pytest.raises(ValueError):
            salt.salt_verify_drafts(ctx, accepted=a, next_token=b, **args)
    big = torch.as_strided(torch.zeros(8, device="cuda"), (1, (1 << 20) + 1), (0, 0))
    with pytest.raises((salt.SaltError, ValueError)):
        salt.salt_verify_drafts(ctx, i32([0, 0]), i32([]), big, q[:0], u[:0], su, a, b)
    torch.cuda.synchronize()
    assert salt.salt_get_device_error(ctx) == 0
