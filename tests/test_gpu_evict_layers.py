"""An eviction in more layers than the plan has room for at a time: its tables are used again within the call."""
import numpy as np
import pytest
import torch

from keeping_reference import evict

pytestmark = pytest.mark.gpu

ARRAYS = ("k", "v", "k_exp", "v_exp", "weights")


@pytest.fixture(scope="module")
def ctx(salt_lib):
    c = salt_lib.salt_ctx_create([64], [64], 1, 1, 1, 1, 1)
    yield c
    salt_lib.salt_ctx_destroy(c)


@pytest.mark.parametrize("kv_heads,max_seqs,dim", [(512, 9000, 64), (512, 3500, 64), (256, 16384, 128)])
@pytest.mark.parametrize("layer,n_layers", [(0, 5), (1, 3)])
def test_parts_of_the_layers(salt_lib, ctx, kv_heads, max_seqs, dim, layer, n_layers):
    """Room for 2^22 chunks, of which each request that the plan may have takes one a head and layer: for one layer, or two, of five."""
    page, layers, lens = 16, 5, [70, 33, 16, 150]
    salt, r = salt_lib, np.random.RandomState(kv_heads)
    need = [-(-n // page) for n in lens]
    ptr = np.cumsum([0] + need).tolist()
    order = r.permutation(ptr[-1] + 1).tolist()
    batch = dict(kv_len=lens, page_ptr=ptr, pages=order[:ptr[-1]])
    shape = (layers, ptr[-1] + 1, kv_heads, page)
    g = torch.Generator(device="cuda").manual_seed(max_seqs)
    rand = lambda s: torch.randint(0, 256, s, dtype=torch.uint8, device="cuda", generator=g)  # noqa: E731
    t = dict(k=rand(shape + (dim,)), v=rand(shape + (dim,)), k_exp=rand(shape), v_exp=rand(shape), weights=torch.randn(shape, device="cuda", generator=g))
    scores = torch.randint(-20, 20, shape, device="cuda", generator=g).float()
    kv = salt.salt_kv_create(ctx, *(t[n] for n in ARRAYS[:4]))
    plan = salt.salt_attn_create(kv, kv_heads, max_seqs, 4, ptr[-1])
    salt.salt_attn_track(plan)
    salt.salt_attn_build(plan, salt.salt_attn_batch([0] * 4, lens, ptr, batch["pages"]))
    keep = [40, 33, 3, 149]
    kept = torch.full((n_layers, 4, kv_heads, 150), -7, dtype=torch.int32, device="cuda")
    before = [t[n].cpu().numpy() for n in ARRAYS]
    salt.salt_attn_evict(plan, layer, n_layers, torch.tensor(keep, dtype=torch.int32, device="cuda"), scores, kept, 2, 10, t["weights"])
    torch.cuda.synchronize()
    arrays, want = evict(before, batch, page, range(layer, layer + n_layers), keep, scores.cpu().numpy(), np.full(tuple(kept.shape), -7), 2, 10)
    assert salt.salt_get_device_error(ctx) == 0
    assert np.array_equal(kept.cpu().numpy(), want)
    for n, a in zip(ARRAYS, arrays):
        assert np.array_equal(t[n].cpu().numpy().view(np.uint8), a.view(np.uint8)), n
