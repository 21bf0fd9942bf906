"""Plain 64-bit definitions of the cached tokens' attention weights and of
eviction (numpy and torch on the CPU, none of the library's code)."""
import math

import numpy as np
import torch

from attn_reference import tokens_of


def lists_of(batch):
    """A batch's lists of cached tokens: (pages, tokens, tokens that were there
    before the step, [(query row, tokens of the list it sees)]) of every request and every group."""
    own, pre = [], []
    rows = {g: [] for g in range(len(batch["group_len"]))}
    at = 0
    for b, n in enumerate(batch["q_len"]):
        kv = batch["kv_len"][b]
        pages = batch["pages"][batch["page_ptr"][b]:batch["page_ptr"][b + 1]]
        own.append((pages, kv, max(0, kv - n), [(at + i, max(0, kv - n + i + 1)) for i in range(n)]))
        if batch["group"][b] >= 0:
            rows[batch["group"][b]] += [at + i for i in range(n)]
        at += n
    for g, n in enumerate(batch["group_len"]):
        pages = batch["group_pages"][batch["group_page_ptr"][g]:batch["group_page_ptr"][g + 1]]
        pre.append((pages, n, n, [(r, n) for r in rows[g]]))
    return own + pre


def add_weights(weights, k_cache, q, lse, batch, page, scale, decay):
    """weights [pages, KV, page] of one layer after a step, in 64 bits, and how far fp32 may be off.  Of a
    score: the query's two terms of 4 bits (2^-22 of its largest element, times sum |k|), fp32 sums of D products (D 2^-23 of sum
    |q k|), its scaling and the difference to the log-sum (2^-22 of both together); of an exponential 2^-20 and
    2^-22 of its argument; of the sum of N terms N 2^-24; of what was there 2^-22.  An exponential below fp32's normal range, 2^-126, may be 0:
2^-126 for each of the N."""
    T, H, D = q.shape
    KV = k_cache.shape[1]
    G = H // KV
    out, tol = weights.double().clone(), torch.zeros(weights.shape, dtype=torch.float64)
    for pages, n, old, rows in lists_of(batch):
        if n == 0 or not rows:
            continue
        K = tokens_of(k_cache, pages, n, page)                       # [n, KV, D]
        r = torch.tensor([i for i, _ in rows])
        see = torch.arange(n)[:, None] < torch.tensor([m for _, m in rows])[None]   # [n, rows]
        if not bool(see.any()):
            continue
        x = q[r].double().view(len(rows), KV, G, D)
        ls = lse[r].double().view(len(rows), KV, G)
        s = torch.einsum("rkgd,nkd->kngr", x, K) * scale
        hide = ~see[None, :, None, :].expand_as(s)
        z = s - ls.permute(1, 2, 0)[:, None]
        p = torch.exp(z.masked_fill(hide, -math.inf))
        ds = abs(scale) * (K.abs().sum(-1).T[:, :, None, None] * x.abs().amax(-1).permute(1, 2, 0)[:, None] * 2.0 ** -22
                           + torch.einsum("rkgd,nkd->kngr", x.abs(), K.abs()) * D * 2.0 ** -23)
        ds = ds + (s.abs() + ls.permute(1, 2, 0)[:, None].abs()) * 2.0 ** -22 + 2.0 ** -20 + z.abs() * 2.0 ** -22
        off = (p * (torch.expm1(ds) + G * len(rows) * 2.0 ** -24)).masked_fill(hide, 0.0).sum((2, 3)).T   # [n, KV]
        total = p.sum((2, 3)).T
        j = torch.arange(n)
        P, O = torch.tensor(pages[:-(-n // page)])[j // page], j % page
        was = weights[P, :, O].double() * decay
        was = torch.where((j < old)[:, None], was, torch.zeros_like(was)) if decay else torch.zeros_like(total)
        seen = see.any(1)
        out[P[seen], :, O[seen]] = (was + total)[seen]
        tol[P[seen], :, O[seen]] = (was.abs() * 2.0 ** -22 + off + total * 2.0 ** -24 + G * len(rows) * 2.0 ** -126)[seen]
    return out, tol


def check_weights(got, want, tol):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan())
    same = (tol == 0) & ~want.isnan()
    assert torch.equal(got[same], want[same])
    err = (got - want).abs() - tol
    bad = ~want.isnan() & ~(err <= 0)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, by {float(err[bad].max()):.3g} over the bound"


def kept_places(scores, keep, first, recent):
    """Places of one line's tokens that are kept, in order."""
    n = len(scores)
    recent = min(recent, keep)
    first = min(first, keep - recent)
    middle = list(range(first, n - recent))
    order = sorted(middle, key=lambda j: (0 if math.isnan(scores[j]) else 1, scores[j] if not math.isnan(scores[j]) else 0.0, -j), reverse=True)
    return sorted(list(range(first)) + order[:keep - first - recent] + list(range(n - recent, n)))


def evict(arrays, batch, page, layers, keep, scores, kept, first, recent):
    """The arrays (numpy, [layers, pages, KV, page, ...]) and kept after an
    eviction in `layers`; an entry of keep outside [0, places] leaves its request."""
    arrays, kept = [a.copy() for a in arrays], kept.copy()
    KV = scores.shape[2]
    for i, l in enumerate(layers):
        for b, n in enumerate(batch["kv_len"]):
            if not 0 <= keep[b] <= kept.shape[3] or keep[b] >= n:
                continue
            pages = np.array(batch["pages"][batch["page_ptr"][b]:batch["page_ptr"][b + 1]], dtype=np.int64)
            j = np.arange(n)
            P, O = pages[j // page], j % page
            for h in range(KV):
                places = np.array(kept_places(scores[l, P, h, O].tolist(), keep[b], first, recent), dtype=np.int64)
                for a in arrays:
                    a[l, P[:keep[b]], h, O[:keep[b]]] = a[l, P[places], h, O[places]]
                kept[i, b, h, :keep[b]] = places
    return arrays, kept
