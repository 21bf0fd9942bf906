"""Plain 64-bit definitions of the cache, attention and draft-verification
operators (numpy and torch on the CPU, none of the library's code), and the
tolerances the tests derive from the kernels' roundings."""
import math

import numpy as np
import torch


# ---------------------------------------------------------------- the cache
def quantise(x):
    """bf16 rows -> (values of the codes, exponent bytes), from the definition."""
    x = x.double()
    finite = torch.isfinite(x).all(-1)
    x = torch.where(finite[..., None], x, torch.zeros_like(x))
    a = x.abs().amax(-1)
    k = torch.full(a.shape, -126, dtype=torch.int64)
    while True:  # the smallest k >= -126 with a <= 448 * 2^k
        up = 448.0 * torch.pow(torch.tensor(2.0, dtype=torch.float64), k.double()) < a
        if not up.any():
            break
        k[up] += 1
    y = x / torch.pow(torch.tensor(2.0, dtype=torch.float64), k.double())[..., None]
    step = torch.pow(torch.tensor(2.0, dtype=torch.float64),
                     torch.clamp(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -30))), min=-6.0) - 3)
    c = torch.round(y / step) * step  # rounds half to even
    e = torch.where(a > 0, k + 127, torch.zeros_like(k))
    e = torch.where(finite, e, torch.full_like(e, 255))
    return c, e


def value(codes, exps):
    """What stored codes and exponent bytes stand for, in 64 bits."""
    c = codes.cpu().view(torch.float8_e4m3fn).double()
    e = exps.cpu().to(torch.int64)
    s = torch.where(e > 0, torch.pow(torch.tensor(2.0, dtype=torch.float64), (e - 127).double()), torch.zeros((), dtype=torch.float64))
    s = torch.where(e == 255, torch.full_like(s, math.nan), s)
    return c * s[..., None]


def tokens_of(x, pages, n, page):
    """[n, heads, dim] rows of a page list of one layer's values [pages, heads, page, dim]."""
    need = -(-n // page)
    if need == 0:
        return x.new_zeros((0, x.shape[1], x.shape[3]))
    return x[torch.tensor(pages[:need])].transpose(1, 2).reshape(-1, x.shape[1], x.shape[3])[:n]


# ---------------------------------------------------------------- attention
def attention(q, k_cache, v_cache, batch, page, scale):
    """q [T, H, D]; caches one layer's values [pages, KV, page, D]; batch: a dict
    of the lengths and page lists.  Returns out, lse and the tolerances of
    both: of out, half a bf16 step of the result (2^-9 |out|), and for each
    probability its rounding to two 4-bit terms (2^-8 at most) and what an
    error of its score makes of it, over sum p |v|; of a score, the
    query's two-term form (2^-17 of its largest element, times sum |k|) and fp32
    sums of D products (D 2^-23 of sum |q k|, at least the 2^-20 of the exponential's argument)."""
    T, H, D = q.shape
    KV = k_cache.shape[1]
    out = torch.zeros((T, H, D), dtype=torch.float64)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, n in enumerate(batch["q_len"]):
        g = batch["group"][b]
        gl = batch["group_len"][g] if g >= 0 else 0
        kv = batch["kv_len"][b]
        own = batch["pages"][batch["page_ptr"][b]:batch["page_ptr"][b + 1]]
        pre = batch["group_pages"][batch["group_page_ptr"][g]:batch["group_page_ptr"][g + 1]] if g >= 0 else []
        kk = torch.cat([tokens_of(k_cache, pre, gl, page), tokens_of(k_cache, own, kv, page)])
        vv = torch.cat([tokens_of(v_cache, pre, gl, page), tokens_of(v_cache, own, kv, page)])
        for i in range(n):
            see = gl + max(0, min(kv, kv - n + i + 1))
            if see == 0:
                continue
            for h in range(H):
                x = q[at + i, h].double()
                K, V = kk[:see, h // (H // KV)], vv[:see, h // (H // KV)]
                s = (K @ x) * scale
                m = s.max()
                p = torch.exp(s - m)
                l = p.sum()
                p = p / l
                o = p @ V
                A = p @ V.abs()
                ds = abs(scale) * ((K.abs().sum(1) * x.abs().max()).max() * 2.0 ** -17 + (K.abs() @ x.abs()).max() * D * 2.0 ** -23)
                ds = ds + s.abs().max() * 2.0 ** -20 + 2.0 ** -20
                out[at + i, h], lse[at + i, h] = o, m + torch.log(l)
                tol[at + i, h] = o.abs() * 2.0 ** -9 + A * (2.0 ** -8 + 2.0 * ds) + 2.0 ** -130
                ltol[at + i, h] = ds + 2.0 ** -18 * (1.0 + lse[at + i, h].abs())
        at += n
    return out, lse, tol, ltol


# ---------------------------------------------------------------- drafts
def units(w):
    w = np.asarray(w, dtype=np.float32)
    w = np.where(w > 0, w, np.float32(0))
    return [int(x) for x in np.floor(np.minimum(w, np.float32(1)).astype(np.float64) * 2.0 ** 40)]


def verify(ptr, tok, p, q, u, su):
    """Whole-number arithmetic of Python; the comparison's product in fp32."""
    accepted, nxt = [], []
    for b in range(len(ptr) - 1):
        n, j = ptr[b + 1] - ptr[b], 0
        while j < n:
            d = ptr[b] + j
            t = tok[d]
            if not (0 <= t < p.shape[1] and np.float32(u[d]) * np.float32(q[d, t]) < p[d + b, t]):
                break
            j += 1
        row = p[ptr[b] + b + j]
        w = units(row - q[ptr[b] + j]) if j < n else units(row)
        if sum(w) == 0:
            w = units(row)
        total = sum(w)
        accepted.append(j)
        if total == 0:
            nxt.append(-1)
            continue
        at = int(np.floor(np.float64(su[b]) * 2 ** 24)) * total >> 24
        run, v = 0, 0
        while True:
            run += w[v]
            if run > at:
                break
            v += 1
        nxt.append(v)
    return accepted, nxt
