"""The operators of a cache whose tokens come and go, whose speed is tracked.

Keys are normalised and rotated to their positions on their way into the paged
8-bit cache, each attention adds to its cached tokens what weight they got, and
a request that has outgrown its share of the cache keeps the tokens that matter.
A case is a dict of plain values; ``kind`` names what one pass does:

* ``rotate``   norms and rotation of a layer's queries and keys, per head: the
               queries as bf16 rows, the keys (and the values as they are) into
               the cache, or both as bf16 rows;
* ``weights``  the attention weights of a batch's cached tokens, summed over
               the rows that see them, added to what was accumulated before;
* ``evict``    all but some cached tokens of each request taken out, for each
               key/value head by itself.

The definitions.  A head x of queries or keys becomes y = x * r * (w + offset),
r = (mean(x^2) + eps)^(-1/2) (without norms y = x), then of its first ``rot``
elements each pair (a, b) turns to (a cos t - b sin t, b cos t + a sin t), t the
token's position times the pair's frequency; pairs are (i, i + rot / 2), or
(2i, 2i + 1) where ``mixed``.  Cached rows are e4m3 codes c and one exponent byte e: with
a = max |y|, k the smallest integer with a <= 448 * 2^k, at least -126, c = y / 2^k
rounded to nearest even and e = k + 127 (e = 0 and c = 0 for a row of zeros).

Row i of a request with n new tokens and L cached tokens of its own (the new ones
among them) sees its domain's whole prompt and its own first L - n + i + 1
tokens.  A cached token's weight is decay * (what it was; 0 for the step's new
tokens) + the sum of exp(scale * q k - lse) over the rows that see it and the query heads
of its key/value head, lse the log-sum of the row's attention.

Eviction leaves a request ``keep`` of its own tokens: the last ``recent``, the first
``first``, and of the others those of the largest scores, ties to the earlier
one.  They move to the front of the request's pages in their order, weights and all; what
lies behind them stays as it was.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0
EPS = 1e-6
THETA = 500000.0


def listed():
    return [
        # one request's new token in one layer of an 8B model, heads normalised: latency
        dict(name="rotate one", kind="rotate", tokens=1, heads=32, kv_heads=8, dim=128, rot=128, mixed=False, norm=True,
             write=True, packed=True, far=10000, page=64),
        # a decode step of 64 requests, far into long documents, heads not normalised
        dict(name="rotate decode", kind="rotate", tokens=64, heads=32, kv_heads=8, dim=128, rot=128, mixed=False, norm=False,
             write=True, packed=True, far=1000000, page=64),
        # a prefill batch, the largest batch the library takes
        dict(name="rotate prefill", kind="rotate", tokens=16384, heads=32, kv_heads=8, dim=128, rot=128, mixed=False, norm=True,
             write=True, packed=True, far=131072, page=64),
        # rows for another attention: half of each head rotated, neighbours as pairs, an odd number of tokens
        dict(name="rotate rows", kind="rotate", tokens=777, heads=24, kv_heads=8, dim=64, rot=32, mixed=True, norm=True,
             write=False, packed=False, far=4096, page=16),
        # one request without a domain prompt decoding one token: latency
        dict(name="weights one", kind="weights", requests=1, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=128, page=64, groups=0,
             prompt=0, own_lo=777, own_hi=777, idle=0.0, decay=1.0),
        # a decode step of 64 requests of four domains
        dict(name="weights shared", kind="weights", requests=64, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=128, page=64, groups=4,
             prompt=4096, own_lo=50, own_hi=1000, idle=0.0, decay=1.0),
        # two requests far into a long document of 64-wide heads, this step's weights by themselves
        dict(name="weights long", kind="weights", requests=2, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=64, page=128, groups=0,
             prompt=0, own_lo=200001, own_hi=262144, idle=0.0, decay=0.0),
        # a prefill chunk of four prompts behind their domain's prompt
        dict(name="weights prompt", kind="weights", requests=4, q_lo=900, q_hi=2048, heads=32, kv_heads=8, dim=128, page=64,
             groups=2, prompt=4096, own_lo=2048, own_hi=4096, idle=0.0, decay=1.0),
        # 48 requests with up to four drafted tokens each, small pages, padding requests among them
        dict(name="weights drafts", kind="weights", requests=48, q_lo=1, q_hi=5, heads=24, kv_heads=8, dim=128, page=16, groups=3,
             prompt=1500, own_lo=1, own_hi=600, idle=0.1, decay=0.9),
        # one request of one layer back to its share of the cache, a page taken out: latency
        dict(name="evict one", kind="evict", requests=1, layers=1, kv_heads=8, dim=128, page=64, own_lo=1088, own_hi=1088,
             keep=1024, first=4, recent=256),
        # 32 requests of some layers of a model, the longer ones cut to three quarters of the longest
        dict(name="evict batch", kind="evict", requests=32, layers=8, kv_heads=8, dim=128, page=64, own_lo=1200, own_hi=2048,
             keep=1536, first=4, recent=512),
        # two long documents cut to a quarter
        dict(name="evict long", kind="evict", requests=2, layers=1, kv_heads=8, dim=64, page=128, own_lo=200001, own_hi=262144,
             keep=65536, first=0, recent=1024),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "weights", "weights", "evict"])
    dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    if kind == "rotate":
        kv_heads = rng.randint(1, 8)
        return dict(kind=kind, tokens=_log_int(rng, 1, 16384), heads=kv_heads * rng.randint(1, 4), kv_heads=kv_heads, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, 16]), mixed=rng.random() < 0.3, norm=rng.random() < 0.5,
                    write=rng.random() < 0.7, packed=rng.random() < 0.5, far=_log_int(rng, 100, 2000000), page=page)
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    if kind == "evict":
        requests, layers = _log_int(rng, 1, 64), rng.randint(1, 8)
        most = min(262144, (1 << 22) // (requests * layers * kv_heads))
        own_hi = _log_int(rng, 16, max(16, most))
        keep = max(1, int(own_hi * rng.uniform(0.05, 0.97)))
        return dict(kind=kind, requests=requests, layers=layers, kv_heads=kv_heads, dim=dim, page=page,
                    own_lo=max(1, own_hi // rng.choice([1, 2, 20])), own_hi=own_hi, keep=keep,
                    first=rng.choice([0, 0, 1, 4, min(keep, 100)]), recent=int(keep * rng.choice([0.0, 0.1, 0.5])))
    shape = rng.choice(["decode", "decode", "drafts", "prompt", "long"])
    c = dict(kind=kind, heads=kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 8] if kv_heads < 8 else [1, 3, 4]), kv_heads=kv_heads, dim=dim,
             page=page, idle=rng.choice([0.0, 0.0, 0.1]), decay=rng.choice([1.0, 1.0, 0.9, 0.0]))
    if shape == "long":
        c.update(requests=rng.randint(1, 2), q_lo=1, q_hi=rng.randint(1, 4), groups=0, prompt=0)
        c["own_hi"] = _log_int(rng, 8192, 262144)
    elif shape == "prompt":
        c.update(requests=rng.randint(1, 4), groups=rng.randint(0, 2), prompt=_log_int(rng, 1, 4096))
        c["q_hi"] = _log_int(rng, 16, 2048)
        c["q_lo"] = max(1, c["q_hi"] // 2)
        c["own_hi"] = c["q_hi"] + rng.choice([0, _log_int(rng, 1, 2048)])
    else:
        c.update(requests=_log_int(rng, 1, 256), groups=rng.randint(0, 8), prompt=_log_int(rng, 1, 8192))
        c["q_hi"] = 1 if shape == "decode" else rng.randint(2, 8)
        c["q_lo"] = 1
        c["own_hi"] = max(c["q_hi"], _log_int(rng, 1, 2000))
    c["own_lo"] = max(c["q_hi"], c["own_hi"] // rng.choice([1, 2, 20]))
    return c


# ---------------------------------------------------------------- layout
def _case_rng(case):
    """A case has the same lengths for every seed, so that its passes do the same work."""
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _batch(case):
    """The lengths of a batch as a scheduler holds them: new and cached tokens
    and the domain of each request, the prompts' lengths."""
    rng, n, G = _case_rng(case), case["requests"], case["groups"]
    q_len = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(n)]
    kv_len = [max(q, rng.randint(case["own_lo"], case["own_hi"])) for q in q_len]
    group = [rng.randrange(G) if G else -1 for _ in range(n)]
    # padding requests of a batch of fixed size: a new token's row, nothing cached, no domain
    idle = [rng.random() < case["idle"] and n > 1 for _ in range(n)]
    q_len, kv_len, group = ([no if i else x for i, x in zip(idle, v)] for v, no in ((q_len, 1), (kv_len, 0), (group, -1)))
    group_len = [max(1, case["prompt"] - rng.randrange(1 + case["prompt"] // 4)) for _ in range(G)]
    return q_len, kv_len, group, group_len


def _evict_lens(case):
    """Each request's cached tokens; the first one has the most."""
    rng = _case_rng(case)
    return [case["own_hi"]] + [rng.randint(case["own_lo"], case["own_hi"]) for _ in range(case["requests"] - 1)]


def _paging(lens, page, first, order):
    """Ragged page lists: (ptr, pages) of as many pages as the lengths need."""
    ptr = [0]
    for n in lens:
        ptr.append(ptr[-1] + -(-n // page))
    return ptr, order[first:first + ptr[-1]], first + ptr[-1]


def _table(ptr, pages, device):
    """The ragged lists as one padded table."""
    n, w = len(ptr) - 1, max([1] + [ptr[i + 1] - ptr[i] for i in range(len(ptr) - 1)])
    t = torch.zeros((max(n, 1), w), dtype=torch.int64)
    for i in range(n):
        if ptr[i + 1] > ptr[i]:
            t[i, :ptr[i + 1] - ptr[i]] = torch.tensor(pages[ptr[i]:ptr[i + 1]])
    return t.to(device)


def _pages_of(slots, page):
    return torch.div(slots, page, rounding_mode="floor"), slots % page


# ---------------------------------------------------------------- plain forms
def _pow2(k):
    """2^k of whole numbers -126 <= k <= 127, made from its bits."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows of x (any shape, last axis a row) -> e4m3 codes and exponent bytes."""
    x = x.float()
    a = x.abs().amax(-1, keepdim=True)
    # a = m * 2^e with m in [0.5, 1), and 448 = 0.875 * 2^9
    m, e = torch.frexp(a)
    k = (torch.where(m <= 0.875, e - 9, e - 8)).clamp(min=-126)
    half = torch.div(k, 2, rounding_mode="floor")  # two factors: 2^-k itself may not be representable
    code = (x * _pow2(-half) * _pow2(half - k)).to(torch.float8_e4m3fn)
    exp = torch.where(a > 0, k + 127, torch.zeros_like(k)).squeeze(-1).to(torch.uint8)
    return code, exp


def _power(e):
    """2^(e - 127) of exponent bytes, 0 for e = 0 (a row of zeros)."""
    return (e.int() << 23).view(torch.float32)


def _plain_rotate(case, x, norm, positions, freq):
    """Heads [tokens, heads, dim] normalised and rotated, in 32 bits; the angles
    in 64, as those of far positions have nothing left of them in 32."""
    y, rot = x.float(), case["rot"]
    if norm is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * norm.float()
    angle = positions.double()[:, None] * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = (y[..., :rot:2], y[..., 1:rot:2]) if case["mixed"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    c, d = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([c, d], -1).flatten(-2) if case["mixed"] else torch.cat([c, d], -1)
    return torch.cat([turned, y[..., rot:]], -1)


def _plain_keys(s, layer, slots):
    """Cached keys [..., heads, dim] of token slots in 32 bits."""
    p, o = _pages_of(slots, s["case"]["page"])
    return s["k"][layer][p, :, o].float() * _power(s["k_exp"][layer][p, :, o]).unsqueeze(-1)


def _plain_slots(table, n, page_tokens):
    p, o = _pages_of(torch.arange(n, device=table.device), page_tokens)
    return table[:, p] * page_tokens + o


def _seen(s, part):
    """The token slots of each request's own tokens or of its domain's prompt,
    [requests, tokens], and which of them each of its rows sees."""
    c, qi = s["case"], torch.arange(s["q_max"], device="cuda")
    live = qi[None, :, None] < s["q_len_d"][:, None, None]
    if part == "own":
        slots = _plain_slots(s["own_table"], max(1, s["own_max"]), c["page"])
        pos = torch.arange(slots.shape[1], device="cuda")
        at = s["kv_len_d"][:, None] - s["q_len_d"][:, None] + qi
        return slots, live & (pos[None, None, :] <= at[:, :, None])
    slots = _plain_slots(s["pre_table"], s["pre_max"], c["page"])[s["group_d"].clamp(min=0)]
    n = torch.where(s["group_d"] >= 0, s["group_len_d"][s["group_d"].clamp(min=0)], 0)
    return slots, live & (torch.arange(slots.shape[1], device="cuda")[None, None, :] < n[:, None, None])


def _scores(s, part):
    """The batch's scores [requests, kv heads, rows, group's heads, tokens], minus infinity where a row does not see a token."""
    c = s["case"]
    H, KV, D, n, qmax = c["heads"], c["kv_heads"], c["dim"], c["requests"], s["q_max"]
    slots, see = _seen(s, part)
    k = _plain_keys(s, 0, slots).permute(0, 2, 3, 1)                                   # [n, KV, D, L]
    q = s["q"][s["row_of"]].float().view(n, qmax, KV, H // KV, D).permute(0, 2, 1, 3, 4).reshape(n, KV, -1, D)
    scores = (q @ k).view(n, KV, qmax, H // KV, -1).mul_(s["scale"])
    return scores.masked_fill_(~see[:, None, :, None, :], -math.inf), slots, see


def _plain_sums(s, part):
    """Each cached token's weight over its request's rows, [requests, kv heads, tokens]."""
    c = s["case"]
    scores, slots, see = _scores(s, part)
    lse = s["lse"][s["row_of"]].view(c["requests"], s["q_max"], c["kv_heads"], -1).permute(0, 2, 1, 3)
    lse = torch.where(lse == -math.inf, torch.zeros_like(lse), lse)
    return scores.sub_(lse[..., None]).exp_().sum((2, 3)), slots, see.any(1)


def _add_weights(s, slots, new, sums, live):
    """weights[slots] = decay * what they were (0 for new tokens) + sums, where live."""
    r, j = live.nonzero(as_tuple=True)
    p, o = _pages_of(slots[r, j], s["case"]["page"])
    w = s["weights"][0]
    old = torch.where(new[r, j][:, None], 0.0, w[p, :, o])
    w[p, :, o] = s["case"]["decay"] * old + sums[r, :, j]


def _plain_weights(s):
    sums, slots, live = _plain_sums(s, "own")
    new = torch.arange(slots.shape[1], device="cuda")[None] >= (s["kv_len_d"] - s["q_len_d"])[:, None]
    _add_weights(s, slots, new, sums, live)
    if s["pre_max"]:
        sums, _, live = _plain_sums(s, "prompt")
        G = s["case"]["groups"]
        both = torch.zeros((G + 1,) + sums.shape[1:], device="cuda")  # (the last one for requests without a domain)
        at = torch.where(s["group_d"] >= 0, s["group_d"], G)
        both.index_add_(0, at, sums)
        lives = torch.zeros((G + 1, live.shape[1]), dtype=torch.int32, device="cuda").index_add_(0, at, live.int())[:G] > 0
        slots = _plain_slots(s["pre_table"], s["pre_max"], s["case"]["page"])
        _add_weights(s, slots, torch.zeros_like(lives), both[:G], lives)
    return s["weights"]


def _evict_places(s):
    """(row numbers of layer, request, head and token place; places kept in order and which of them are any)."""
    c = s["case"]
    P, KV, n_pages = c["page"], c["kv_heads"], s["n_pages"]
    slots = _plain_slots(s["own_table"], s["own_max"], P)
    p, o = _pages_of(slots, P)                                                            # [n, L]
    layer, head = torch.arange(c["layers"], device="cuda"), torch.arange(KV, device="cuda")
    page = (layer[:, None, None, None] * n_pages + p[None, :, None, :]) * KV + head[None, None, :, None]
    rows = page * P + o[None, :, None, :]                                                 # [layers, n, KV, L]
    pos = torch.arange(slots.shape[1], device="cuda")
    n, keep = s["kv_len_d"][:, None], s["keep"].long()[:, None]
    recent = keep.clamp(max=c["recent"])
    first = (keep - recent).clamp(max=c["first"])
    held = (pos >= n - recent) | (pos < first)                                            # [n, L]
    score = s["scores"].flatten()[rows].double()
    score = score.masked_fill(held[None, :, None], math.inf).masked_fill((pos >= n)[None, :, None], -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices[..., :c["keep"]]
    evicted = (keep < n)[None, :, None] & (torch.arange(order.shape[-1], device="cuda") < keep)[None, :, None]
    return rows, torch.where(evicted, order, slots.shape[1]).sort(-1).values, evicted


def _plain_evict(s):
    rows, places, evicted = _evict_places(s)
    src = rows.gather(-1, places.clamp(max=rows.shape[-1] - 1))[evicted.expand_as(places)]
    dst = rows[..., :places.shape[-1]][evicted.expand_as(places)]
    D = s["case"]["dim"]
    for x, w in (("k", D), ("v", D), ("k_exp", 1), ("v_exp", 1)):
        t = s[x].view(torch.uint8).view(-1, w)
        t[dst] = t[src]
    t = s["weights"].view(-1)
    t[dst] = t[src]
    kept = s["kept"][..., :places.shape[-1]]
    kept.copy_(torch.where(evicted, places, kept))


# ---------------------------------------------------------------- states
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(shape, g):
    """Keys or values as projections give them: normal, rows of different
    sizes, a few channels larger than the others."""
    x = torch.randn(shape, generator=g, device="cuda")
    x *= torch.exp(0.4 * torch.randn(shape[:-1] + (1,), generator=g, device="cuda"))
    x[..., ::17] *= 3.0
    return x.to(torch.bfloat16)


def _cache(layers, pages, heads, page, dim, g):
    """A cache in use: every page holds rows, the free ones old ones."""
    kv = []
    for _ in range(2):
        codes = torch.empty((layers, pages, heads, page, dim), dtype=torch.float8_e4m3fn, device="cuda")
        exps = torch.empty((layers, pages, heads, page), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 26) // (heads * page * dim))
        for l in range(layers):
            for a in range(0, pages, step):
                c, e = _quantise(_rows((min(step, pages - a), heads, page, dim), g))
                codes[l, a:a + step] = c
                exps[l, a:a + step] = e
        kv += [codes, exps]
    return dict(k=kv[0], k_exp=kv[1], v=kv[2], v_exp=kv[3])


def _accumulated(shape, g):
    """Weights that tokens gathered over some steps: a few have most of it, some never got any."""
    w = torch.exp(1.5 * torch.randn(shape, generator=g, device="cuda") - 2.0)
    return w * (torch.rand(shape, generator=g, device="cuda") > 0.05)


_context = None


def _library():
    """The library and the one context that a program keeps."""
    global _context
    from paper_2608_03579_gb300 import salt
    if _context is None:
        _context = salt.salt_ctx_create([4096], [4096], 1, 1, 1, 1, 1)
    return salt, _context


def _handle(s):
    salt, ctx = _library()
    s["kv"] = salt.salt_kv_create(ctx, s["k"], s["v"], s["k_exp"], s["v_exp"])


def _plan(s, heads, host):
    salt, _ = _library()
    _handle(s)
    q_len, _, _, own_pages, _, group_len, _, pre_pages = host
    s["plan"] = salt.salt_attn_create(s["kv"], heads, max_seqs=len(q_len), max_tokens=max(1, sum(q_len)),
                                      max_pages=max(1, len(own_pages) + len(pre_pages)), max_groups=max(1, len(group_len)))
    salt.salt_attn_track(s["plan"])
    salt.salt_attn_build(s["plan"], salt.salt_attn_batch(*host))  # once a step, for every layer of it


def prepare(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    return {"rotate": _prepare_rotate, "weights": _prepare_weights, "evict": _prepare_evict}[case["kind"]](case, g, rng)


def _prepare_rotate(case, g, rng):
    T, H, KV, D, P = (case[x] for x in ("tokens", "heads", "kv_heads", "dim", "page"))
    s = {"case": case}
    s["inv_freq"] = [THETA ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]
    s["freq_d"] = torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
    # a few runs of tokens of requests, each from a place of its own
    run = max(1, T // 8)
    start = torch.tensor([rng.randrange(case["far"]) for _ in range(-(-T // run))], device="cuda")
    s["positions"] = (start.repeat_interleave(run)[:T] + torch.arange(T, device="cuda") % run).int()
    if case["packed"]:  # as slices of the rows of a fused q/k/v projection
        qkv = _rows((T, H + 2 * KV, D), g)
        s["q"], s["new_k"], s["new_v"] = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    else:
        s["q"], s["new_k"], s["new_v"] = _rows((T, H, D), g), _rows((T, KV, D), g), _rows((T, KV, D), g)
    s["q_norm"], s["k_norm"] = ((1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16) if case["norm"] else None
                                for _ in range(2))
    s["q_out"] = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
    if case["write"]:
        pages = -(-T // P) + 3
        s.update(_cache(1, pages, KV, P, D, g))
        order = torch.randperm(pages, generator=g, device="cuda")
        p, o = _pages_of(torch.arange(T, device="cuda"), P)
        s["slots"] = (order[p] * P + o).int()
    else:
        s["k_out"] = torch.empty((T, KV, D), dtype=torch.bfloat16, device="cuda")
    if own:
        salt, ctx = _library()
        s["rope"] = salt.salt_rope_create(ctx, D, case["rot"], s["inv_freq"], interleaved=case["mixed"], eps=EPS)
        if case["write"]:
            _handle(s)
    return s


def _prepare_weights(case, g, rng):
    P, D = case["page"], case["dim"]
    q_len, kv_len, group, group_len = _batch(case)
    n_pages = sum(-(-n // P) for n in kv_len) + sum(-(-n // P) for n in group_len) + 5
    order = list(range(n_pages))
    rng.shuffle(order)
    pre_ptr, pre_pages, nxt = _paging(group_len, P, 0, order)
    own_ptr, own_pages, _ = _paging(kv_len, P, nxt, order)
    s = {"case": case, "scale": D ** -0.5, **_cache(1, n_pages, case["kv_heads"], P, D, g)}
    T = sum(q_len)
    s["q"] = torch.randn((T, case["heads"], D), generator=g, device="cuda").to(torch.bfloat16)
    s["weights"] = _accumulated((1, n_pages, case["kv_heads"], P), g)
    s["host"] = (q_len, kv_len, own_ptr, own_pages, group, group_len, pre_ptr, pre_pages)
    # the same lengths and pages as arrays on the GPU
    s["q_max"], s["own_max"], s["pre_max"] = max(q_len), max(kv_len), max(group_len, default=0)
    s["q_len_d"], s["kv_len_d"], s["group_d"] = (torch.tensor(v, device="cuda") for v in (q_len, kv_len, group))
    s["group_len_d"] = torch.tensor(group_len or [0], device="cuda")
    s["own_table"], s["pre_table"] = _table(own_ptr, own_pages, "cuda"), _table(pre_ptr, pre_pages, "cuda")
    q_ptr = s["q_len_d"].cumsum(0) - s["q_len_d"]
    s["row_of"] = q_ptr[:, None] + torch.minimum(torch.arange(s["q_max"], device="cuda"), s["q_len_d"][:, None] - 1)
    # the log-sums that the attention left
    lse = torch.logsumexp(_scores(s, "own")[0], -1)
    if s["pre_max"]:
        lse = torch.logaddexp(lse, torch.logsumexp(_scores(s, "prompt")[0], -1))
    b = torch.repeat_interleave(torch.arange(len(q_len), device="cuda"), s["q_len_d"])
    s["lse"] = lse.permute(0, 2, 1, 3).reshape(len(q_len), s["q_max"], -1)[b, torch.arange(T, device="cuda") - q_ptr[b]].contiguous()
    if own:
        _plan(s, case["heads"], s["host"])
    return s


def _prepare_evict(case, g, rng):
    P, D, KV, L = case["page"], case["dim"], case["kv_heads"], case["layers"]
    kv_len = _evict_lens(case)
    n = len(kv_len)
    n_pages = sum(-(-x // P) for x in kv_len) + 3
    order = list(range(n_pages))
    rng.shuffle(order)
    ptr, pages, _ = _paging(kv_len, P, 0, order)
    s = {"case": case, "n_pages": n_pages, **_cache(L, n_pages, KV, P, D, g)}
    s["weights"] = _accumulated((L, n_pages, KV, P), g)
    s["scores"] = s["weights"].clone()  # what goes by the accumulated weights (a program may smooth them)
    s["keep"] = torch.tensor([min(x, case["keep"]) for x in kv_len], dtype=torch.int32, device="cuda")
    s["kept"] = torch.full((L, n, KV, case["keep"]), -1, dtype=torch.int32, device="cuda")
    s["own_max"], s["own_table"] = max(kv_len), _table(ptr, pages, "cuda")
    s["kv_len_d"] = torch.tensor(kv_len, device="cuda")
    if own:
        _plan(s, KV, ([1] * n, kv_len, ptr, pages, [-1] * n, [], [0], []))
    return s


# ---------------------------------------------------------------- passes
def _cached(s):
    """The cache's codes, and the powers of two that its exponent bytes stand for."""
    return [s["k"], s["k_exp"].view(torch.float8_e8m0fnu), s["v"], s["v_exp"].view(torch.float8_e8m0fnu)]


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2608_03579_gb300 import salt
    c = s["case"]
    if c["kind"] == "rotate":
        if not c["write"]:
            salt.salt_rope_apply(s["rope"], s["q"], s["new_k"], s["positions"], s["q_out"], s["k_out"], s["q_norm"], s["k_norm"])
            return [s["q_out"], s["k_out"]]
        salt.salt_rope_write(s["rope"], s["kv"], 0, s["q"], s["new_k"], s["new_v"], s["positions"], s["slots"], s["q_out"],
                             s["q_norm"], s["k_norm"])
        return [s["q_out"]] + _cached(s)
    if c["kind"] == "weights":
        salt.salt_attn_weights(s["plan"], 0, s["q"], s["lse"], s["scale"], s["weights"], decay=c["decay"])
        return [s["weights"]]
    salt.salt_attn_evict(s["plan"], 0, c["layers"], s["keep"], s["scores"], s["kept"], first=c["first"], recent=c["recent"],
                         weights=s["weights"])
    return [s["k"], s["k_exp"], s["v"], s["v_exp"], s["weights"], s["kept"]]


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "rotate":
        s["q_out"].copy_(_plain_rotate(c, s["q"], s["q_norm"], s["positions"], s["freq_d"]))
        k = _plain_rotate(c, s["new_k"], s["k_norm"], s["positions"], s["freq_d"])
        if not c["write"]:
            s["k_out"].copy_(k)
            return [s["q_out"], s["k_out"]]
        p, o = _pages_of(s["slots"].long(), c["page"])
        for x, y in (("k", k), ("v", s["new_v"])):
            codes, exps = _quantise(y)
            s[x][0].view(torch.uint8)[p, :, o] = codes.view(torch.uint8)
            s[x + "_exp"][0][p, :, o] = exps
        return [s["q_out"]] + _cached(s)
    if c["kind"] == "weights":
        return [_plain_weights(s)]
    _plain_evict(s)
    return [s["k"], s["k_exp"], s["v"], s["v_exp"], s["weights"], s["kept"]]


# ---------------------------------------------------------------- work
def work(case):
    """Bytes and operations of one pass; a domain's prompt is read once, not
    once a request."""
    kind, D, KV = case["kind"], case["dim"], case["kv_heads"]
    if kind == "rotate":
        T, H = case["tokens"], case["heads"]
        kv = KV * 2 * (3 * D + 1) if case["write"] else KV * 4 * D
        return {"bytes": T * (H * 4 * D + kv + (8 if case["write"] else 4)), "flops": T * (H + KV) * D * 10}
    if kind == "evict":
        moved = places = 0
        for n in _evict_lens(case):
            if n > case["keep"]:
                # every kept row but those before the first that goes is read and written
                moved += case["layers"] * KV * max(0, case["keep"] - case["first"])
                places += case["layers"] * KV * n
        left = case["requests"] * 4
        return {"bytes": left + places * 4 + moved * (2 * (2 * D + 2 + 4) + 4), "flops": 0}
    q_len, kv_len, group, group_len = _batch(case)
    H = case["heads"]
    used = {g for g in group if g >= 0}
    tokens = sum(kv_len) + sum(group_len[g] for g in used)
    pairs = 0
    for q, kv, g in zip(q_len, kv_len, group):
        first = kv - q + 1  # own tokens that the first row sees
        pairs += sum(max(0, first + i) for i in range(q)) + (q * group_len[g] if g >= 0 else 0)
    return {"bytes": tokens * KV * (D + 1 + (8 if case["decay"] else 4)) + sum(q_len) * H * (2 * D + 4), "flops": 2 * pairs * H * D}


# ---------------------------------------------------------------- 64 bits
def _exact_pow2(k):
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """The values the stored codes stand for in units of their power of two,
    and that power of two (2^-127 for a row of zeros), from the definition."""
    x = x.double()
    a = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(a.clamp(min=1e-300) / E4M3_MAX))
    k = torch.where(E4M3_MAX * _exact_pow2(k - 1) >= a, k - 1, k)
    k = torch.where(E4M3_MAX * _exact_pow2(k) < a, k + 1, k).clamp(min=-126)
    y = x / _exact_pow2(k)
    least = y.abs().clamp(min=2.0 ** -6)
    binade = torch.floor(torch.log2(least))
    binade = torch.where(_exact_pow2(binade) > least, binade - 1, binade)
    binade = torch.where(_exact_pow2(binade + 1) <= least, binade + 1, binade)
    step = _exact_pow2(binade - 3)
    return torch.round(y / step) * step, _exact_pow2(torch.where(a > 0, k, torch.full_like(k, -127.0))).squeeze(-1)


def _exact_turned(case, x, norm, at, freq):
    """Complex numbers turned by their angle, pair by pair."""
    x, rot = x.double(), case["rot"]
    if norm is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * norm.double()
    pair = torch.arange(rot // 2, device="cuda")
    i, j = (2 * pair, 2 * pair + 1) if case["mixed"] else (pair, pair + rot // 2)
    angle = at.double()[:, None] * freq
    z = torch.complex(x[..., i], x[..., j]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    x = x.clone()
    x[..., i], x[..., j] = z.real, z.imag
    return x


def _exact_rotate(s):
    c = s["case"]
    q = _exact_turned(c, s["q"], s["q_norm"], s["positions"], s["freq_d"])
    k = _exact_turned(c, s["new_k"], s["k_norm"], s["positions"], s["freq_d"])
    if not c["write"]:
        return [q, k]
    p, o = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
    res = [q]
    for x, y in (("k", k), ("v", s["new_v"])):
        codes, power = s[x].double(), _exact_pow2(s[x + "_exp"].long() - 127)
        codes[0][p, :, o], power[0][p, :, o] = _exact_rows(y)
        res += [codes, power]
    return res


def exact(case, seed):
    if case["kind"] == "evict":
        return None  # whole numbers, and values that are moved as they are
    s = prepare(case, seed)
    if case["kind"] == "rotate":
        return _exact_rotate(s)
    P, H, KV, D = case["page"], case["heads"], case["kv_heads"], case["dim"]
    q_len, kv_len, own_ptr, own_pages, group, group_len, pre_ptr, pre_pages = s["host"]
    if sum(q * (kv + case["prompt"]) for q, kv in zip(q_len, kv_len)) * H * (2 * D + 50) > 6e12:
        return None
    w = s["weights"][0].double()
    # the decayed old weights first, then request by request what its rows add
    used = sorted({g for g in group if g >= 0})
    lists = [(own_pages[own_ptr[b]:own_ptr[b + 1]], kv_len[b], max(0, kv_len[b] - q_len[b])) for b in range(len(q_len))]
    lists += [(pre_pages[pre_ptr[g]:pre_ptr[g + 1]], group_len[g], group_len[g]) for g in used]
    for pages, n, old in lists:
        if n:
            j = torch.arange(n, device="cuda")
            p, o = torch.tensor(pages, device="cuda")[j // P], j % P
            w[p, :, o] = torch.where((j < old)[:, None], w[p, :, o] * case["decay"], 0.0)
    at = 0
    for b, n in enumerate(q_len):
        for own_part in (True, False):
            g = group[b]
            if (own_part and not kv_len[b]) or (not own_part and g < 0):
                continue
            pages, m = lists[b][:2] if own_part else (pre_pages[pre_ptr[g]:pre_ptr[g + 1]], group_len[g])
            j = torch.arange(m, device="cuda")
            p, o = torch.tensor(pages, device="cuda")[j // P], j % P
            e = s["k_exp"][0][p, :, o]
            k = s["k"][0][p, :, o].double() * torch.where(e > 0, _exact_pow2(e.long() - 127), 0.0)[..., None]
            for i0 in range(0, n, 256):
                i = torch.arange(i0, min(n, i0 + 256), device="cuda")
                q = s["q"][at + i].double().view(len(i), KV, H // KV, D)
                sc = torch.einsum("ikgd,lkd->kgil", q, k) * s["scale"]
                p_row = torch.exp(sc - s["lse"][at + i].double().view(len(i), KV, H // KV).permute(1, 2, 0)[..., None])
                if own_part:
                    p_row = p_row.masked_fill(~(j[None, :] <= (kv_len[b] - n + i)[:, None]), 0.0)
                w[p, :, o] += p_row.sum((1, 2)).T
        at += n
    return [w[None]]
