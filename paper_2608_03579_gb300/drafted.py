"""Generation with drafted tokens for requests that share their domain's prompt.

A small decoder with random weights that runs the library's calls as a serving
program does.  Each domain's prompt goes through the model once, adapted by the
domain's centroid alone, so that its cached keys and values hold for every
user of the domain.  A step then takes the last token of every
request and the tokens that a cheap model drafted after it:

    salt_build_segments, salt_attn_build         once a step
    salt_lora_apply_with_base                    q | k | v of a layer, centroid and residual
    salt_kv_write                                the k and v columns, as they lie
    salt_attn_run                                the q columns, over prompt and own tokens
    salt_verify_drafts                           once a step

A rejected draft's cached rows are not taken out: the request's length just stays
behind them and the next step writes over them.

    python -m paper_2608_03579_gb300.drafted
"""
from __future__ import annotations

import numpy as np
import torch

from . import salt
from .runner import bf16_bits


class Request:
    def __init__(self, domain: int, user: int, first_token: int, pages):
        self.domain, self.user, self.pages = domain, user, pages
        self.tokens = [first_token]   # the last one is not in the cache yet
        self.cached = 0


class DraftedDecoder:
    def __init__(self, layers=2, hidden=512, heads=8, kv_heads=2, head_dim=64, vocab=1000, domains=2, rank=16, users=6,
                 page_tokens=16, pages=128, pages_per_request=8, max_tokens=256, max_requests=16, seed=0):
        self.n_layers, self.heads, self.kv_heads, self.head_dim, self.page_tokens = layers, heads, kv_heads, head_dim, page_tokens
        self.vocab, self.pages_per_request = vocab, pages_per_request
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        width = (heads + 2 * kv_heads) * head_dim
        d_in, d_out = [hidden] * layers, [width] * layers
        self.ctx = salt.salt_ctx_create(d_in, d_out, domains, rank, users, 2, max_tokens, torch.cuda.current_device())
        self.seg = salt.salt_segments_create(self.ctx)
        for d in range(domains):
            salt.salt_centroid_pin(self.ctx, d, rank, self._normal(layers * rank * hidden, hidden ** -0.5),
                                   self._normal(layers * rank * width, rank ** -0.5), 0.5)
        for u in range(users):
            r = 1 + u % 2
            a, b = self._normal(layers * r * hidden, hidden ** -0.5), self._normal(layers * r * width, 1.0)
            blob = torch.empty(salt.salt_residual_blob_bytes(d_in, d_out, r), dtype=torch.uint8, pin_memory=True)
            salt.salt_residual_blob_pack(d_in, d_out, r, 0.5, bf16_bits(a), bf16_bits(b), blob.numpy(), blob.numel())
            salt.salt_residual_load(self.ctx, u, blob)
            torch.cuda.current_stream().synchronize()   # the blob may go
        self.embed = self._normal((vocab, hidden), 1.0)
        self.w_qkv = [self._normal((hidden, width), hidden ** -0.5) for _ in range(layers)]
        self.w_o = [self._normal((heads * head_dim, hidden), hidden ** -0.5) for _ in range(layers)]
        self.w_out = self._normal((hidden, vocab), 2.0 * hidden ** -0.5)
        # the drafting model knows the last token only
        self.draft_p = torch.softmax((self.embed @ self.w_out).float(), -1)
        shape = (layers, pages, kv_heads, page_tokens, head_dim)
        byte = dict(dtype=torch.uint8, device="cuda")
        self.cache = (torch.empty(shape, **byte), torch.empty(shape, **byte), torch.empty(shape[:4], **byte), torch.empty(shape[:4], **byte))
        self.kv = salt.salt_kv_create(self.ctx, *self.cache)
        self.attn = salt.salt_attn_create(self.kv, heads, max_requests, max_tokens, pages, domains)
        self.free = list(range(pages))
        self.prompts = [[] for _ in range(domains)]   # a domain's prompt tokens and their pages
        self.prompt_pages = [[] for _ in range(domains)]
        self.requests: list[Request] = []

    def _normal(self, shape, scale):
        n = (shape,) if isinstance(shape, int) else shape
        return (torch.randn(n, generator=self.gen, device="cuda") * scale).bfloat16()

    def close(self):
        salt.salt_attn_destroy(self.attn)
        salt.salt_kv_destroy(self.kv)
        salt.salt_segments_destroy(self.seg)
        salt.salt_ctx_destroy(self.ctx)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    def _pages(self, tokens: int):
        n = -(-tokens // self.page_tokens)
        if n > len(self.free):
            raise RuntimeError("the cache is full")
        return [self.free.pop() for _ in range(n)]

    def _slots(self, pages, start: int, n: int):
        return [pages[j // self.page_tokens] * self.page_tokens + j % self.page_tokens for j in range(start, start + n)]

    def _forward(self, tokens, dom, user, slots, batch, seen=None):
        """Probabilities after each token, [tokens, vocab]; seen(layer, q, out) looks on."""
        cuda = dict(device="cuda")
        H, KV, D, T = self.heads, self.kv_heads, self.head_dim, tokens.numel()
        salt.salt_build_segments(self.ctx, self.seg, np.asarray(dom, np.int32), np.asarray(user, np.int32))
        salt.salt_attn_build(self.attn, batch)
        slots = torch.tensor(slots, dtype=torch.int32, **cuda)
        x = self.embed[tokens]
        for l in range(self.n_layers):
            y = torch.empty((T, (H + 2 * KV) * D), dtype=torch.bfloat16, **cuda)
            salt.salt_lora_apply_with_base(self.ctx, self.seg, l, x, self.w_qkv[l], salt.SALT_W_IN_OUT, y)
            rows = y.view(T, H + 2 * KV, D)
            q, k, v = rows[:, :H], rows[:, H:H + KV], rows[:, H + KV:]
            salt.salt_kv_write(self.kv, l, k, v, slots)
            o = torch.empty((T, H, D), dtype=torch.bfloat16, **cuda)
            salt.salt_attn_run(self.attn, l, q, o, D ** -0.5)
            if seen is not None:
                seen(l, q, o)
            x = x.float() + (o.view(T, H * D) @ self.w_o[l]).float()
            x = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).bfloat16()
        return torch.softmax((x @ self.w_out).float(), -1)

    def set_prompts(self, prompts, seen=None):
        """Each domain's prompt (lists of tokens) through the model and into the cache."""
        lens = [len(p) for p in prompts]
        pages = [self._pages(n) for n in lens]
        self.prompts, self.prompt_pages = [list(p) for p in prompts], pages
        dom = [d for d, n in enumerate(lens) for _ in range(n)]
        batch = dict(q_len=lens, kv_len=lens, page_ptr=np.cumsum([0] + [len(p) for p in pages]).tolist(), pages=sum(pages, []))
        look = None if seen is None else lambda l, q, o: seen(l, q, o, batch)
        tokens = torch.tensor(sum(self.prompts, []), dtype=torch.int64, device="cuda")
        if tokens.numel():
            self._forward(tokens, dom, [-1] * len(dom), sum((self._slots(p, 0, n) for p, n in zip(pages, lens)), []),
                          salt.salt_attn_batch(**batch), look)

    def add(self, domain: int, user: int, first_token: int):
        self.requests.append(Request(domain, user, first_token, self._pages(self.pages_per_request * self.page_tokens)))

    def step(self, drafts, seen=None) -> dict:
        """One step; drafts[b]: how many tokens to draft for request b.  Returns what was verified."""
        cuda = dict(device="cuda")
        room = [r.pages and len(r.pages) * self.page_tokens - r.cached for r in self.requests]
        if any(n + 1 > m for n, m in zip(drafts, room)):
            raise RuntimeError("a request's pages are full")
        ptr = np.cumsum([0] + list(drafts))
        # drafted one after the other, every request's next one together
        last = torch.tensor([r.tokens[-1] for r in self.requests], **cuda)
        drawn = [last]
        for _ in range(max(drafts, default=0)):
            drawn.append(torch.multinomial(self.draft_p[drawn[-1]], 1, generator=self.gen).flatten())
        drawn = torch.stack(drawn).cpu().numpy()                     # [1 + most drafts][requests]
        fed = [drawn[:n + 1, b] for b, n in enumerate(drafts)]       # what a request puts through the model
        tokens = torch.as_tensor(np.concatenate(fed), **cuda)
        q_rows = self.draft_p[torch.as_tensor(np.concatenate([f[:-1] for f in fed]), **cuda)]
        draft_tokens = torch.as_tensor(np.concatenate([f[1:] for f in fed]).astype(np.int32), **cuda)
        q_len = [n + 1 for n in drafts]
        kv_len = [r.cached + n for r, n in zip(self.requests, q_len)]
        batch = dict(q_len=q_len, kv_len=kv_len, page_ptr=np.cumsum([0] + [len(r.pages) for r in self.requests]).tolist(),
                     pages=sum((r.pages for r in self.requests), []), group=[r.domain for r in self.requests],
                     group_len=[len(p) for p in self.prompts],
                     group_page_ptr=np.cumsum([0] + [len(p) for p in self.prompt_pages]).tolist(),
                     group_pages=sum(self.prompt_pages, []))
        look = None if seen is None else lambda l, q, o: seen(l, q, o, batch)
        slots = sum((self._slots(r.pages, r.cached, n) for r, n in zip(self.requests, q_len)), [])
        dom = [r.domain for r, n in zip(self.requests, q_len) for _ in range(n)]
        user = [r.user for r, n in zip(self.requests, q_len) for _ in range(n)]
        p = self._forward(tokens, dom, user, slots, salt.salt_attn_batch(**batch), look)
        n = len(self.requests)
        u, su = (torch.rand(k, generator=self.gen, **cuda) for k in (int(ptr[-1]), n))
        accepted, following = (torch.empty(n, dtype=torch.int32, **cuda) for _ in range(2))
        salt.salt_verify_drafts(self.ctx, torch.as_tensor(ptr.astype(np.int32), **cuda), draft_tokens, p, q_rows, u, su, accepted, following)
        done = dict(ptr=ptr.tolist(), tokens=draft_tokens, p=p, q=q_rows, u=u, su=su, accepted=accepted.tolist(), next=following.tolist())
        for r, f, a, t in zip(self.requests, fed, done["accepted"], done["next"]):
            r.tokens += f[1:1 + a].tolist() + [t]
            r.cached += 1 + a
        return done


def main():
    with DraftedDecoder() as m:
        host = np.random.RandomState(0)
        m.set_prompts([host.randint(0, m.vocab, n).tolist() for n in (150, 37)])
        for b in range(6):
            m.add(b % 2, b, int(host.randint(m.vocab)))
        drafted = accepted = 0
        for _ in range(8):
            done = m.step([3, 0, 4, 2, 5, 1])
            drafted += done["ptr"][-1]
            accepted += sum(done["accepted"])
        assert salt.salt_get_device_error(m.ctx) == 0
        for r in m.requests:
            print(f"domain {r.domain}, user {r.user}: {r.tokens}")
        print(f"{accepted} of {drafted} drafted tokens accepted in 8 steps of {len(m.requests)} requests")


if __name__ == "__main__":
    main()
