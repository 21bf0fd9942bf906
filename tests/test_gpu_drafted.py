"""The library's calls run together as a serving program runs them: adapted
projections, cache writes, attention over shared prompts and draft verification,
each step's attention and decisions against the 64-bit definitions."""
import numpy as np
import pytest
import torch

from attn_reference import attention, value, verify

pytestmark = pytest.mark.gpu


@pytest.fixture
def drafted(salt_lib):
    from paper_2608_03579_gb300 import drafted
    return drafted


def make(drafted, lens, seed=0, **kw):
    m = drafted.DraftedDecoder(seed=seed, **kw)
    host = np.random.RandomState(seed)
    watched = []

    def seen(layer, q, out, batch):
        full = dict(group=[-1] * len(batch["q_len"]), group_len=[], group_page_ptr=[0], group_pages=[]) | batch
        k, v, ke, ve = (t[layer] for t in m.cache)
        ref, _, tol, _ = attention(q.cpu(), value(k, ke), value(v, ve), full, m.page_tokens, m.head_dim ** -0.5)
        far = (out.cpu().double() - ref).abs() - tol
        assert far.max() <= 0, (layer, far.max())
        watched.append(layer)

    m.set_prompts([host.randint(0, m.vocab, n).tolist() for n in lens], seen)
    return m, host, seen, watched


@pytest.mark.parametrize("lens, page, dim", [((70, 33), 16, 64), ((0, 129), 64, 128)])
def test_steps_against_the_definitions(drafted, lens, page, dim):
    m, host, seen, watched = make(drafted, lens, page_tokens=page, head_dim=dim, heads=4, kv_heads=2, pages_per_request=max(2, 64 // page))
    with m:
        for b in range(5):
            m.add(b % 2, b, int(host.randint(m.vocab)))
        for counts in ([2, 0, 3, 1, 4], [0, 0, 0, 0, 0], [5, 1, 0, 2, 3]):
            before = [(list(r.tokens), r.cached) for r in m.requests]
            d = m.step(counts, seen)
            ref_a, ref_n = verify(d["ptr"], d["tokens"].cpu().numpy(), d["p"].cpu().numpy(), d["q"].cpu().numpy(),
                                  d["u"].cpu().numpy(), d["su"].cpu().numpy())
            assert (d["accepted"], d["next"]) == (ref_a, ref_n)
            for r, (old, cached), a, t in zip(m.requests, before, ref_a, ref_n):
                assert r.cached == cached + a + 1 == len(r.tokens) - 1
                assert r.tokens[:len(old)] == old and r.tokens[-1] == t and 0 <= t < m.vocab
        assert m.n_layers * 3 <= len(watched)
        from paper_2608_03579_gb300 import salt
        assert salt.salt_get_device_error(m.ctx) == 0


def test_same_seed_same_tokens(drafted):
    runs = []
    for _ in range(2):
        m, host, _, _ = make(drafted, (40, 90), seed=3)
        with m:
            for b in range(4):
                m.add(b % 2, b, int(host.randint(m.vocab)))
            for _ in range(4):
                m.step([3, 1, 0, 2])
            runs.append([r.tokens for r in m.requests])
    assert runs[0] == runs[1]


def test_full_pages_are_refused(drafted):
    m, _, _, _ = make(drafted, (5, 5), pages_per_request=1)
    with m:
        m.add(0, 0, 1)
        with pytest.raises(RuntimeError, match="full"):
            m.step([16])


def test_main_runs(drafted, capsys):
    drafted.main()
    assert "drafted tokens accepted" in capsys.readouterr().out


def test_other_types_are_refused(salt_lib, drafted):
    m, _, _, _ = make(drafted, (5, 5))
    with m:
        rows = lambda t: torch.zeros((2, m.kv_heads, m.head_dim), dtype=t, device="cuda")
        slots = torch.full((2,), -1, dtype=torch.int32, device="cuda")
        bf, half = rows(torch.bfloat16), rows(torch.float16)
        for k, v in ((half, bf), (bf, half)):
            with pytest.raises(ValueError):
                salt_lib.salt_kv_write(m.kv, 0, k, v, slots)
            with pytest.raises(ValueError):
                salt_lib.salt_kv_read(m.kv, 0, slots, k, v)
        salt_lib.salt_attn_build(m.attn, salt_lib.salt_attn_batch([1], [0], [0, 0], []))
        q = torch.zeros((1, m.heads, m.head_dim), dtype=torch.bfloat16, device="cuda")
        with pytest.raises(ValueError):
            salt_lib.salt_attn_run(m.attn, 0, q.half(), q, 1.0)
        with pytest.raises(ValueError):
            salt_lib.salt_attn_run(m.attn, 0, q, q.clone(), 1.0, lse=torch.zeros((1, m.heads), dtype=torch.int32, device="cuda"))
        ints = torch.zeros(2, dtype=torch.int32, device="cuda")
        p = torch.zeros((2, 8), device="cuda")
        args = lambda p, u: (m.ctx, ints, ints[:1], p, p[:1], u, u, ints[:1], ints[1:])
        with pytest.raises(ValueError):
            salt_lib.salt_verify_drafts(*args(p.int(), p[0, :1].contiguous()))
        with pytest.raises(ValueError):
            salt_lib.salt_verify_drafts(*args(p, ints[:1]))


def test_verification_without_a_context(salt_lib):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    p = torch.tensor([[0.5, 0.25, 0.25, 0.0], [0.0, 0.0, 1.0, 0.0]], device="cuda")
    q = torch.tensor([[0.25, 0.75, 0.0, 0.0]], device="cuda")
    u, su = torch.tensor([0.5], device="cuda"), torch.tensor([0.0], device="cuda")
    a, b = i32([9]), i32([9])
    for token, accepted, following in ((0, 1, 2), (1, 0, 0), (7, 0, 0)):  # 7: outside the vocabulary
        salt_lib.salt_verify_drafts(None, i32([0, 1]), i32([token]), p, q, u, su, a, b)
        assert (a.item(), b.item()) == (accepted, following)
    with pytest.raises(salt_lib.SaltError):
        salt_lib.salt_verify_drafts(None, i32([0, 0]), i32([]), torch.zeros((1, (1 << 20) + 4), device="cuda"), q[:0], u[:0], su, a, b)
