"""What the calls on a tracked plan refuse without a GPU, and the tests' own
definitions on small cases."""
import ctypes
import math

import numpy as np
import pytest
import torch

from keeping_reference import add_weights, evict, kept_places


def test_null_handles(salt_lib):
    lib = salt_lib._lib
    assert lib.salt_attn_track(None) == 1
    assert lib.salt_attn_weights(None, 0, None, 0, None, 1.0, 1.0, None, None) == 1
    assert lib.salt_attn_evict(None, 0, 1, None, 0, 0, None, None, None, ctypes.c_int64(0), None) == 1


def test_tensors_are_checked_before_the_call(salt_lib):
    salt_lib._load_types()
    kv, plan = object.__new__(salt_lib.KvCache), object.__new__(salt_lib.AttnPlan)
    kv.handle = plan.handle = plan.ctx = None
    kv.rows_shape, kv.n_kv_heads = torch.Size((1, 2, 2, 16)), 2
    plan.kv, plan.n_heads, plan.head_dim, plan.n_tokens, plan.n_seqs = kv, 4, 64, 3, 1
    q, lse, w = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 4)), torch.zeros((1, 2, 2, 16))
    with pytest.raises(ValueError):
        salt_lib.salt_attn_weights(plan, 0, q, lse, 1.0, w)                                         # host tensors
    keep, kept = torch.zeros(1, dtype=torch.int32), torch.zeros((1, 1, 2, 5), dtype=torch.int32)
    for args in ((keep, w, kept), (keep, w, kept[:, :, :1]), (keep, w, kept[0])):
        with pytest.raises(ValueError):
            salt_lib.salt_attn_evict(plan, 0, 1, *args)


def test_kept_places():
    s = [3.0, 1.0, 2.0, 2.0, math.nan, -math.inf, 2.0, 0.5]
    assert kept_places(s, 3, 0, 0) == [0, 2, 3]
    assert kept_places(s, 3, 0, 1) == [0, 2, 7]
    assert kept_places(s, 4, 2, 1) == [0, 1, 2, 7]
    assert kept_places(s, 4, 9, 9) == [4, 5, 6, 7]
    assert kept_places(s, 4, 9, 1) == [0, 1, 2, 7]
    assert kept_places(s, 7, 0, 0) == [0, 1, 2, 3, 5, 6, 7]
    assert kept_places(s, 0, 3, 3) == []
    assert kept_places([0.0, -0.0, 0.0], 2, 0, 0) == [0, 1]


def test_eviction_of_a_line():
    scores = np.array([5, 1, 4, 3, 9, 9], dtype=np.float32).reshape(1, 3, 1, 2)       # three pages of two tokens
    batch = dict(kv_len=[5], page_ptr=[0, 3], pages=[2, 0, 1])
    x = np.arange(6).reshape(1, 3, 1, 2)
    kept = np.full((1, 1, 1, 4), -1)
    # tokens in order: 9 9 5 1 4; the last one and the two largest
    (y,), kept = evict([x], batch, 2, [0], [3], scores, kept, 0, 1)
    assert kept.tolist() == [[[[0, 1, 4, -1]]]]
    assert y.reshape(-1).tolist() == [2, 1, 2, 3, 4, 5]


def test_weights_of_one_row():
    """A row's weights are its probabilities; decay and the step's own token."""
    K = torch.randn((2, 1, 16, 64), dtype=torch.float64)
    q = torch.randn((1, 1, 64)).bfloat16()
    batch = dict(q_len=[1], kv_len=[20], page_ptr=[0, 2], pages=[1, 0], group=[-1], group_len=[], group_page_ptr=[0], group_pages=[])
    k = torch.cat([K[1, 0], K[0, 0, :4]])
    s = k @ q[0, 0].double() * 0.125
    lse = torch.logsumexp(s, 0).view(1, 1)
    was = torch.rand((2, 1, 16))
    got, tol = add_weights(was, K, q, lse, batch, 16, 0.125, 0.5)
    p = torch.softmax(s, 0)
    assert torch.allclose(got[1, 0], p[:16] + 0.5 * was[1, 0].double()) and torch.allclose(got[0, 0, :3], p[16:19] + 0.5 * was[0, 0, :3].double())
    assert torch.allclose(got[0, 0, 3], p[19]) and torch.equal(got[0, 0, 4:], was[0, 0, 4:].double())
    assert bool((tol[0, 0, 4:] == 0).all()) and bool((tol[1] > 0).all()) and bool((tol[1] < 1e-3).all())
