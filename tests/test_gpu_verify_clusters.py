"""Verification where a request's CTAs cannot all start at once: runs on several
streams beside other work, over vocabularies that take one to eight CTAs a
request, good draft pointers and bad ones side by side."""
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


@pytest.mark.parametrize("V", [2000, 2049, 8000, 16385, 40000])
def test_clusters_beside_other_work(salt_lib, ctx, V):
    n, r = 60, np.random.RandomState(V)
    d = r.randint(0, 4, n)
    ptr = [0] + np.cumsum(d).tolist()
    D = ptr[-1]
    p, q = (r.exponential(size=(k, V)).astype(np.float32) for k in (D + n, D))
    p, q = p / p.sum(1, keepdims=True), q / q.sum(1, keepdims=True)
    tok, u, su = r.randint(0, V, D), r.rand(D).astype(np.float32), r.rand(n).astype(np.float32)
    want = verify(ptr, tok.tolist(), p, q, u, su)
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()  # noqa: E731
    args = (f(np.asarray(ptr, np.int32)), f(tok.astype(np.int32)), f(p), f(q), f(u), f(su))
    busy = torch.randn((2048, 2048), device="cuda")
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    done = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 4]):
            if i % 4 == 0:
                busy = busy @ busy * 1e-2
            res = torch.full((2, n), 77, dtype=torch.int32, device="cuda")
            salt_lib.salt_verify_drafts(ctx, *args, res[0], res[1])
            done.append(res)
    torch.cuda.synchronize()
    for res in done:
        assert (res[0].tolist(), res[1].tolist()) == tuple(want)
    assert salt_lib.salt_get_device_error(ctx) == 0


def test_bad_pointers_among_good_ones(salt_lib, ctx):
    """A request whose pointers are out of order ends its CTAs early, the others' go on."""
    V = 20000
    p, q = torch.full((6, V), 1 / V, device="cuda"), torch.full((3, V), 1 / V, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    a, b = i32([9] * 3), i32([9] * 3)
    salt_lib.salt_verify_drafts(ctx, i32([0, 1, 0, 1]), i32([V, 5, 5]), p, q, torch.ones(3, device="cuda"),
                                torch.full((3,), 0.1, device="cuda"), a, b)
    torch.cuda.synchronize()
    w = 1 << 40
    first = int(np.floor(np.float64(np.float32(0.1)) * 2 ** 24)) * (V * int(np.float32(1 / V) * w)) >> 24
    token = first // int(np.float32(1 / V) * w)
    assert a.tolist() == [0, 0, 0] and b.tolist() == [token, -1, token]
    assert salt_lib.salt_get_device_error(ctx) == 0x200
