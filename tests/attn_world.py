"""Batches whose requests all read the same cached tokens, so that many rows and
long items cost little memory, and their 64-bit attention on the GPU (torch's
float64, none of the library's code)."""
import math

import numpy as np
import torch

from attn_reference import quantise, value


def bf16_rows(n, kv_heads, dim, seed, spread=0.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, kv_heads, dim), generator=g) * torch.exp(spread * torch.randn((n, kv_heads, 1), generator=g))).bfloat16()


class Shared:
    """Every request's own tokens are k[prompt:], v[prompt:] (the first kv_len
    of them), behind k[:prompt], v[:prompt] as its group's prompt if there is one.
    Pages in a shuffled order; what lies past the lengths is NaN codes and
    wild exponents."""

    def __init__(self, salt, ctx, k, v, q_len, kv_len, heads, page=64, prompt=0, seed=0, scale=None):
        n, kv_heads, dim = k.shape
        self.salt, self.ctx, self.heads, self.kv_heads, self.dim, self.page, self.prompt = salt, ctx, heads, kv_heads, dim, page, prompt
        self.q_len, self.kv_len, self.T = list(q_len), list(kv_len), sum(q_len)
        need = [-(-prompt // page), -(-(n - prompt) // page)]
        order = np.random.RandomState(seed).permutation(sum(need) + 2).tolist()
        self.lists = [order[:need[0]], order[need[0]:sum(need)]]
        shape = (1, len(order), kv_heads, page, dim)
        self.codes, self.exps, self.values = {}, {}, {}
        pos = torch.arange(n)
        pos = torch.where(pos < prompt, pos, pos - prompt + need[0] * page)  # the own list starts on a page
        pages, offset = torch.tensor(order)[pos // page], pos % page
        for name, x in (("k", k), ("v", v)):
            c = torch.full(shape, 0x7F, dtype=torch.uint8)
            e = torch.full(shape[:4], 254 if name == "k" else 255, dtype=torch.uint8)
            qc, qe = quantise(x)
            c[0, pages, :, offset] = qc.to(torch.float8_e4m3fn).view(torch.uint8)
            e[0, pages, :, offset] = qe.to(torch.uint8)
            self.codes[name], self.exps[name] = c.cuda(), e.cuda()
            self.values[name] = value(c[0, pages, :, offset], e[0, pages, :, offset]).cuda()
        self.unit = torch.where(qe == 255, torch.zeros(()), torch.exp2(qe.double() - 127)).cuda()   # of the values' codes [n, KV]
        g = torch.Generator().manual_seed(seed + 1)
        self.q = torch.randn((self.T, heads, dim), generator=g).bfloat16().cuda()
        self.scale = dim ** -0.5 if scale is None else scale
        self.kv = salt.salt_kv_create(ctx, self.codes["k"], self.codes["v"], self.exps["k"], self.exps["v"])
        R = len(self.q_len)
        self.plan = salt.salt_attn_create(self.kv, heads, R, max(1, self.T), need[0] + R * need[1] + 1, 1)

    def build(self, stream=None):
        R, own = len(self.q_len), len(self.lists[1])
        grouped = self.prompt > 0
        self.salt.salt_attn_build(self.plan, self.salt.salt_attn_batch(
            self.q_len, self.kv_len, [own * i for i in range(R + 1)], self.lists[1] * R, [0 if grouped else -1] * R,
            [self.prompt] if grouped else [], [0, len(self.lists[0])] if grouped else [0], self.lists[0] if grouped else []), stream)

    def run(self, stream=None):
        out = torch.full((self.T, self.heads, self.dim), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.T, self.heads), 7.0, device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.salt.salt_attn_run(self.plan, 0, self.q, out, self.scale, lse, stream)
        torch.cuda.synchronize()
        assert self.salt.salt_get_device_error(self.ctx) == 0
        return out, lse

    def requests(self):
        """(rows, cached values K and V, which of them each row sees) of each request."""
        at = 0
        for n, kv in zip(self.q_len, self.kv_len):
            keep = self.prompt + kv
            K, V = (self.values[x][:keep] for x in "kv")
            j, i = torch.arange(keep, device="cuda"), torch.arange(n, device="cuda")
            yield slice(at, at + n), K, V, j[None] < self.prompt + torch.clamp(kv - n + i + 1, min=0)[:, None]
            at += n

    def reference(self):
        """out, lse and their tolerances: those of attn_reference.attention, row by row, and for out
        the end of f16's range, in which probabilities times their value's power of two meet the
        values' codes: the largest of a row is at least 2^2 and all are rounded by 2^-25 at least."""
        G, D = self.heads // self.kv_heads, self.dim
        f64 = dict(dtype=torch.float64, device="cuda")
        out, tol = torch.zeros((self.T, self.heads, D), **f64), torch.zeros((self.T, self.heads, D), **f64)
        lse, ltol = torch.full((self.T, self.heads), -math.inf, **f64), torch.zeros((self.T, self.heads), **f64)
        for at, K, V, see in self.requests():
            n, keep = see.shape
            if keep == 0:
                continue
            x = self.q[at].double().view(n, self.kv_heads, G, D)
            hide = ~see[:, None, None]
            s = torch.einsum("nkgd,tkd->nkgt", x, K) * self.scale
            none = hide.all(-1)
            ls = torch.logsumexp(s.masked_fill(hide, -math.inf), -1)
            p = torch.exp(s.masked_fill(hide, -math.inf) - torch.where(none, torch.zeros_like(ls), ls)[..., None])
            o, A = torch.einsum("nkgt,tkd->nkgd", p, V), torch.einsum("nkgt,tkd->nkgd", p, V.abs())
            most = lambda t: t.masked_fill(hide, 0.0).amax(-1)  # noqa: E731
            ksum = K.abs().sum(-1).T[None, :, None]                                # [1, KV, 1, t]
            ds = abs(self.scale) * (most(ksum.expand_as(s)) * x.abs().amax(-1) * 2.0 ** -17
                                    + most(torch.einsum("nkgd,tkd->nkgt", x.abs(), K.abs())) * D * 2.0 ** -23)
            ds = ds + most(s.abs()) * 2.0 ** -20 + 2.0 ** -20
            unit = self.unit[:keep]
            codes = (V.abs() / torch.where(unit > 0, unit, torch.ones_like(unit))[..., None]).nan_to_num(0.0).sum(0)   # [KV, D]
            least = (p * unit.T[None, :, None]).amax(-1)[..., None] * codes[None, :, None] * 2.0 ** -27
            out[at], lse[at] = o.reshape(n, -1, D), ls.reshape(n, -1)
            tol[at] = (o.abs() * 2.0 ** -9 + A * (2.0 ** -8 + 2.0 * ds)[..., None] + least + 2.0 ** -130).reshape(n, -1, D)
            ltol[at] = (ds + 2.0 ** -18 * (1.0 + ls.abs())).reshape(n, -1)
        return out, lse, tol, ltol


def compare(got, glse, out, lse, tol, ltol):
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(glse), empty) and bool((glse[empty] < 0).all())
    assert bool((got[empty] == 0).all())
    err = (got.double() - out).abs() - tol
    assert bool((err <= 0).all()), f"out off by {float(err.max()):.3g} over its bound"
    lerr = torch.where(empty, torch.zeros_like(lse), (glse.double() - lse).abs() - ltol)
    assert bool((lerr <= 0).all()), f"lse off by {float(lerr.max()):.3g} over its bound"
