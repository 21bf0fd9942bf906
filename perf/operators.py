"""The serving operators around the adapted projections whose speed is tracked.

A decoder layer's q/k/v projections are followed by three things: the new keys
and values go into the cache, the queries attend to it, and at the step's end
the tokens a draft model proposed are held against the target's probabilities.
A case is a dict of plain values; ``kind`` names what one pass does:

* ``write``   new keys and values into a paged cache of 8-bit floats;
* ``read``    cached keys and values back as bf16;
* ``attn``    attention of a batch whose requests share their domain's prompt,
              reading that cache;
* ``step``    the cache part of a serving step: the plan of the batch, then for
              each layer the write of its new tokens and the attention;
* ``verify``  drafted tokens accepted or replaced.

The definitions.  A cached row (one token, one head) x of bf16 is stored as
e4m3 codes c and one exponent byte e: with a = max |x|, k the smallest integer
with a <= 448 * 2^k, at least -126, c = x / 2^k rounded to nearest even and
e = k + 127 (e = 0 and c = 0 for a row of zeros); it stands for c * 2^k.
Attention row i of a request with n new tokens and L cached tokens of its own
(the new ones among them) sees its domain's whole prompt and its own first
L - n + i + 1 tokens; a row that sees nothing gives zeros and a log-sum of
minus infinity.  A drafted token t is accepted while u * q(t) < p(t); at the
first that is not, the next token is drawn from max(p - q, 0), after the last
from p, by inverting the running sum of the weights in units of 2^-40.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0


def listed():
    return [
        # a decode step's new tokens of one layer of an 8B model (64 requests): latency
        dict(name="write decode", kind="write", tokens=64, heads=8, dim=128, page=64, packed=True),
        # a prefill batch's tokens, the largest batch the library takes
        dict(name="write prefill", kind="write", tokens=16384, heads=8, dim=128, page=64, packed=True),
        # one request's cache moved out of the pool
        dict(name="read request", kind="read", tokens=777, heads=8, dim=64, page=16),
        # a long context's cache, for a layer that wants bf16
        dict(name="read long", kind="read", tokens=100003, heads=8, dim=128, page=128),
        # one request without a domain prompt decoding one token: latency
        dict(name="decode one", kind="attn", requests=1, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=128, page=64, groups=0,
             prompt=0, own_lo=777, own_hi=777, idle=0.0, lse=False),
        # decoding 64 requests of four domains
        dict(name="decode shared", kind="attn", requests=64, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=128, page=64, groups=4,
             prompt=4096, own_lo=50, own_hi=1000, idle=0.0, lse=False),
        # 48 requests of a 3B model with up to four drafted tokens each, small pages, padding requests among them
        dict(name="drafts shared", kind="attn", requests=48, q_lo=1, q_hi=5, heads=24, kv_heads=8, dim=128, page=16, groups=3,
             prompt=1500, own_lo=1, own_hi=600, idle=0.1, lse=True),
        # two requests far into a long document of 64-wide heads
        dict(name="decode long", kind="attn", requests=2, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=64, page=128, groups=0,
             prompt=0, own_lo=200001, own_hi=262144, idle=0.0, lse=True),
        # a prefill chunk of four prompts behind their domain's prompt
        dict(name="prompt chunk", kind="attn", requests=4, q_lo=900, q_hi=2048, heads=32, kv_heads=8, dim=128, page=64, groups=2,
             prompt=4096, own_lo=2048, own_hi=4096, idle=0.0, lse=False),
        # a decode step of 256 requests of eight domains: plan, cache writes and attention of two layers
        dict(name="step full", kind="step", requests=256, q_lo=1, q_hi=1, heads=32, kv_heads=8, dim=128, page=64, groups=8,
             prompt=8192, own_lo=100, own_hi=2000, idle=0.0, lse=False, layers=2),
        # one request's four drafted tokens: latency
        dict(name="verify one", kind="verify", requests=1, d_lo=4, d_hi=4, vocab=32000, gap=1.0),
        # a full batch's drafts over a large vocabulary
        dict(name="verify full", kind="verify", requests=256, d_lo=0, d_hi=7, vocab=131072, gap=0.5),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "attn", "attn", "attn", "step", "verify"])
    dim, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    if kind == "write":
        return dict(kind=kind, tokens=_log_int(rng, 1, 16384), heads=rng.randint(1, 8), dim=dim, page=page,
                    packed=rng.random() < 0.5)
    if kind == "read":
        return dict(kind=kind, tokens=_log_int(rng, 1, 100000), heads=rng.randint(1, 8), dim=dim, page=page)
    if kind == "verify":
        d_hi = rng.randint(0, 7)
        return dict(kind=kind, requests=_log_int(rng, 1, 256), d_lo=rng.randint(0, d_hi), d_hi=d_hi,
                    vocab=_log_int(rng, 100, 131072), gap=round(rng.uniform(0.0, 3.0), 3))
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 5, 8])
    shape = rng.choice(["decode", "drafts", "prompt", "long"]) if kind == "attn" else "decode"
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, dim=dim, page=page, idle=rng.choice([0.0, 0.0, 0.1]),
             lse=rng.random() < 0.5)
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
    if kind == "step":
        c["layers"] = rng.randint(1, 2)
    return c


# ---------------------------------------------------------------- layout
def _batch(case):
    """The lengths of a batch as a scheduler holds them: new and cached tokens
    and the domain of each request, the prompts' lengths.  A case has the same
    ones for every seed, so that its passes do the same work."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    n, G = case["requests"], case["groups"]
    q_len = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(n)]
    kv_len = [max(q, rng.randint(case["own_lo"], case["own_hi"])) for q in q_len]
    group = [rng.randrange(G) if G else -1 for _ in range(n)]
    # padding requests of a batch of fixed size: a new token's row, nothing cached, no domain
    for b in range(n):
        if rng.random() < case["idle"] and n > 1:
            q_len[b], kv_len[b], group[b] = 1, 0, -1
    group_len = [max(1, case["prompt"] - rng.randrange(1 + case["prompt"] // 4)) for _ in range(G)]
    return q_len, kv_len, group, group_len


def _paging(lens, page, first, order):
    """Ragged page lists: (ptr, pages) of as many pages as the lengths need."""
    ptr, pages = [0], []
    for n in lens:
        k = -(-n // page)
        pages += order[first:first + k]
        first += k
        ptr.append(len(pages))
    return ptr, pages, first


def _table(ptr, pages, device):
    """The ragged lists as one padded table."""
    n, w = len(ptr) - 1, max([1] + [ptr[i + 1] - ptr[i] for i in range(len(ptr) - 1)])
    t = torch.zeros((max(n, 1), w), dtype=torch.int64)
    for i in range(n):
        if ptr[i + 1] > ptr[i]:
            t[i, :ptr[i + 1] - ptr[i]] = torch.tensor(pages[ptr[i]:ptr[i + 1]])
    return t.to(device)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- plain forms
def _pow2(k):
    """2^k of whole numbers -126 <= k <= 127, made from its bits."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows of x (any shape, last axis a row) -> e4m3 codes and exponent bytes."""
    x = x.float()
    a = x.abs().amax(-1, keepdim=True)
    # bf16 rows: a = m * 2^e with 8 bits of m in [0.5, 1), and 448 = 0.875 * 2^9
    m, e = torch.frexp(a)
    k = (torch.where(m <= 0.875, e - 9, e - 8)).clamp(min=-126)
    half = torch.div(k, 2, rounding_mode="floor")  # two factors: 2^-k itself may not be representable
    code = (x * _pow2(-half) * _pow2(half - k)).to(torch.float8_e4m3fn)
    exp = torch.where(a > 0, k + 127, torch.zeros_like(k)).squeeze(-1).to(torch.uint8)
    return code, exp


def _power(e):
    """2^(e - 127) of exponent bytes, 0 for e = 0 (a row of zeros)."""
    return (e.int() << 23).view(torch.float32)


def _plain_write(codes, exps, x, page, offset):
    c, e = _quantise(x)
    codes.view(torch.uint8)[page, :, offset] = c.view(torch.uint8)
    exps[page, :, offset] = e


def _plain_rows(codes, exps, slots, page_tokens):
    """Cached rows [..., heads, dim] of token slots in 32 bits."""
    p, o = torch.div(slots, page_tokens, rounding_mode="floor"), slots % page_tokens
    return codes[p, :, o].float() * _power(exps[p, :, o]).unsqueeze(-1)


def _plain_slots(table, n, page_tokens):
    pos = torch.arange(n, device=table.device)
    return table[:, torch.div(pos, page_tokens, rounding_mode="floor")] * page_tokens + pos % page_tokens


def _plain_attn(s, layer):
    c = s["case"]
    P, H, KV, D = c["page"], c["heads"], c["kv_heads"], c["dim"]
    n, qmax, lown, lpre = c["requests"], s["q_max"], max(1, s["own_max"]), s["pre_max"]
    # each request's tokens: its domain's prompt, then its own
    own_slots = _plain_slots(s["own_table"], lown, P)
    pos = torch.arange(lown, device="cuda")
    at = s["kv_len_d"][:, None] - s["q_len_d"][:, None] + torch.arange(qmax, device="cuda")
    see = pos[None, None, :] <= at[:, :, None]
    see &= pos[None, None, :] < s["kv_len_d"][:, None, None]
    slots = own_slots
    if lpre:
        pre = _plain_slots(s["pre_table"], lpre, P)[s["group_d"].clamp(min=0)]
        slots = torch.cat([pre, own_slots], 1)
        plen = torch.where(s["group_d"] >= 0, s["group_len_d"][s["group_d"].clamp(min=0)], 0)
        pv = torch.arange(lpre, device="cuda")[None, None, :] < plen[:, None, None]
        see = torch.cat([pv.expand(n, qmax, lpre), see], 2)
    k = _plain_rows(s["k"][layer], s["k_exp"][layer], slots, P).permute(0, 2, 3, 1)     # [n, KV, D, L]
    v = _plain_rows(s["v"][layer], s["v_exp"][layer], slots, P).permute(0, 2, 1, 3)     # [n, KV, L, D]
    qi = torch.arange(qmax, device="cuda")
    row = s["q_ptr_d"][:-1, None] + torch.minimum(qi, (s["q_len_d"][:, None] - 1).clamp(min=0))
    q = s["q"][layer][row].float().view(n, qmax, KV, H // KV, D).permute(0, 2, 1, 3, 4).reshape(n, KV, -1, D)
    scores = (q @ k).view(n, KV, qmax, H // KV, -1) * s["scale"]
    scores = scores.masked_fill(~see[:, None, :, None, :], -math.inf)
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(m == -math.inf, torch.zeros_like(m), m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    o = (p.view(n, KV, -1, p.shape[-1]) @ v).view(n, KV, qmax, H // KV, D).permute(0, 2, 1, 3, 4).reshape(n, qmax, H, D)
    lse = (m + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(n, qmax, H)
    b, i = s["token_at"]  # the batch's tokens in order, without the padding
    return o[b, i].to(torch.bfloat16), lse[b, i]


def _plain_verify(s):
    p_all, q_all, tok, u = s["target"], s["draft"], s["tokens"].long(), s["accept_u"]
    ptr = s["ptr"].long()
    n = ptr[1:] - ptr[:-1]
    b = torch.arange(len(n), device="cuda")
    j = torch.arange(max(1, s["case"]["d_hi"]), device="cuda")
    have = j[None, :] < n[:, None]
    d = (ptr[:-1, None] + j).clamp(max=max(0, len(tok) - 1))
    if len(tok):
        t = tok[d]
        ok = (u[d] * q_all[d, t] < p_all[d + b[:, None], t]) & have
    else:
        ok = have & False
    accepted = torch.cumprod(ok.int(), 1).sum(1)
    p = p_all[ptr[:-1] + b + accepted]
    if len(tok):
        q = q_all[(ptr[:-1] + accepted).clamp(max=len(tok) - 1)]
        q = torch.where((accepted < n)[:, None], q, torch.zeros_like(q))
    else:
        q = torch.zeros_like(p)

    def units(w):
        return (torch.where(w > 0, w, torch.zeros_like(w)).clamp(max=1.0) * 2.0 ** 40).to(torch.int64)

    w = units(p - q)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, units(p))  # p nowhere above q: p itself
    run_sum = torch.cumsum(w, 1)
    total = run_sum[:, -1]
    uu = (s["sample_u"] * 2.0 ** 24).to(torch.int64)
    at = uu * (total >> 24) + ((uu * (total & 0xFFFFFF)) >> 24)
    token = (run_sum <= at[:, None]).sum(1)
    return accepted.int(), torch.where(total > 0, token, -1).int()


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


def prepare(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    s = {"case": case}
    if case["kind"] == "verify":
        return _prepare_verify(case, s, g, rng)
    P, D = case["page"], case["dim"]
    if case["kind"] in ("write", "read"):
        T, H = case["tokens"], case["heads"]
        pages = -(-T // P) + 3
        s.update(_cache(1, pages, H, P, D, g))
        order = torch.randperm(pages, generator=g, device="cuda")
        pos = torch.arange(T, device="cuda")
        s["slots"] = (order[torch.div(pos, P, rounding_mode="floor")] * P + pos % P).int()
        if case["kind"] == "write":
            if case["packed"]:  # as slices of the rows of a fused q/k/v projection
                qkv = _rows((T, 6 * H, D), g)
                s["new_k"], s["new_v"] = qkv[:, 4 * H:5 * H], qkv[:, 5 * H:]
            else:
                s["new_k"], s["new_v"] = _rows((T, H, D), g), _rows((T, H, D), g)
        else:
            s["out_k"] = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
            s["out_v"] = torch.empty_like(s["out_k"])
        if own:
            _handle(s)
        return s
    q_len, kv_len, group, group_len = _batch(case)
    layers = case.get("layers", 1)
    n_pages = sum(-(-n // P) for n in kv_len) + sum(-(-n // P) for n in group_len) + 5
    order = list(range(n_pages))
    rng.shuffle(order)
    pre_ptr, pre_pages, nxt = _paging(group_len, P, 0, order)
    own_ptr, own_pages, _ = _paging(kv_len, P, nxt, order)
    s.update(_cache(layers, n_pages, case["kv_heads"], P, D, g))
    T = sum(q_len)
    s["scale"] = D ** -0.5
    s["q"] = [torch.randn((T, case["heads"], D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(layers)]
    s["out"] = [torch.empty_like(q) for q in s["q"]]
    s["lse"] = torch.empty((T, case["heads"]), device="cuda") if case["lse"] else None
    s["host"] = (q_len, kv_len, own_ptr, own_pages, group, group_len, pre_ptr, pre_pages)
    q_ptr = [0]
    for n in q_len:
        q_ptr.append(q_ptr[-1] + n)
    if case["kind"] == "step":
        H = case["kv_heads"]
        slots = []
        for b, n in enumerate(q_len):  # the new tokens are the last of the cached ones (a padding request has none)
            for i in range(n):
                t = kv_len[b] - n + i
                slots.append(own_pages[own_ptr[b] + t // P] * P + t % P if t >= 0 else -1)
        s["slots"] = _i32(slots)
        s["new"] = [(_rows((T, H, D), g), _rows((T, H, D), g)) for _ in range(layers)]
    if own:
        salt, _ = _library()
        _handle(s)
        s["plan"] = salt.salt_attn_create(s["kv"], case["heads"], max_seqs=case["requests"], max_tokens=max(T, 1),
                                          max_pages=max(1, len(own_pages) + len(pre_pages)),
                                          max_groups=max(1, len(group_len)))
        s["batch"] = salt.salt_attn_batch(*s["host"])
        if case["kind"] == "attn":  # one plan serves every layer of a step
            salt.salt_attn_build(s["plan"], s["batch"])
        return s
    # the same lengths and pages as arrays on the GPU
    s["q_max"], s["own_max"], s["pre_max"] = max(q_len), max(kv_len), max(group_len, default=0)
    s["q_len_d"], s["kv_len_d"] = (torch.tensor(v, device="cuda") for v in (q_len, kv_len))
    s["q_ptr_d"], s["group_d"] = (torch.tensor(v, device="cuda") for v in (q_ptr, group))
    s["group_len_d"] = torch.tensor(group_len or [0], device="cuda")
    s["own_table"] = _table(own_ptr, own_pages, "cuda")
    s["pre_table"] = _table(pre_ptr, pre_pages, "cuda")
    b = torch.repeat_interleave(torch.arange(len(q_len)), torch.tensor(q_len))
    s["token_at"] = (b.cuda(), (torch.arange(T) - torch.tensor(q_ptr)[b]).cuda())
    return s


def _prepare_verify(case, s, g, rng):
    n, V = case["requests"], case["vocab"]
    d = [rng.randint(case["d_lo"], case["d_hi"]) for _ in range(n)]
    ptr = [0]
    for x in d:
        ptr.append(ptr[-1] + x)
    D = ptr[-1]
    logits = 2.0 * torch.randn((D + n, V), generator=g, device="cuda")
    s["target"] = torch.softmax(logits, -1)
    at = [ptr[b] + b + j for b in range(n) for j in range(d[b])]
    at = torch.tensor(at, dtype=torch.int64, device="cuda")
    logits = logits[at]
    logits += case["gap"] * torch.randn((D, V), generator=g, device="cuda")  # the draft model's idea of the same rows
    s["draft"] = torch.softmax(logits, -1)
    # drafted from q, as a draft model does
    s["tokens"] = (s["draft"] / torch.empty_like(logits).exponential_(generator=g)).argmax(-1).int() if D else _i32([])
    s["ptr"] = _i32(ptr)
    s["accept_u"] = torch.rand(D, generator=g, device="cuda")
    s["sample_u"] = torch.rand(n, generator=g, device="cuda")
    s["accepted"], s["next"] = (torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(2))
    return s


# ---------------------------------------------------------------- passes
def _state_out(s):
    return [s["k"], s["k_exp"], s["v"], s["v_exp"]]


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2608_03579_gb300 import salt
    case = s["case"]
    kind = case["kind"]
    if kind == "write":
        salt.salt_kv_write(s["kv"], 0, s["new_k"], s["new_v"], s["slots"])
        return _state_out(s)
    if kind == "read":
        salt.salt_kv_read(s["kv"], 0, s["slots"], s["out_k"], s["out_v"])
        return [s["out_k"], s["out_v"]]
    if kind == "attn":
        salt.salt_attn_run(s["plan"], 0, s["q"][0], s["out"][0], s["scale"], lse=s["lse"])
        return [s["out"][0]] + ([s["lse"]] if case["lse"] else [])
    if kind == "step":
        salt.salt_attn_build(s["plan"], s["batch"])
        for l in range(case["layers"]):
            salt.salt_kv_write(s["kv"], l, s["new"][l][0], s["new"][l][1], s["slots"])
            salt.salt_attn_run(s["plan"], l, s["q"][l], s["out"][l], s["scale"], lse=s["lse"])
        return s["out"] + ([s["lse"]] if case["lse"] else []) + _state_out(s)
    salt.salt_verify_drafts(_context, s["ptr"], s["tokens"], s["target"], s["draft"], s["accept_u"], s["sample_u"],
                            s["accepted"], s["next"])
    return [s["accepted"], s["next"]]


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "write":
        p, o = torch.div(s["slots"], case["page"], rounding_mode="floor").long(), (s["slots"] % case["page"]).long()
        _plain_write(s["k"][0], s["k_exp"][0], s["new_k"], p, o)
        _plain_write(s["v"][0], s["v_exp"][0], s["new_v"], p, o)
        return _state_out(s)
    if kind == "read":
        slots = s["slots"].long()
        return [_plain_rows(s[x][0], s[x + "_exp"][0], slots, case["page"]).to(torch.bfloat16) for x in ("k", "v")]
    if kind == "attn":
        o, lse = _plain_attn(s, 0)
        return [o] + ([lse] if case["lse"] else [])
    if kind == "step":
        outs, lse = [], None
        keep = (s["slots"] >= 0).nonzero().squeeze(1)  # a padding request's row goes nowhere
        slots = s["slots"][keep]
        p, o = torch.div(slots, case["page"], rounding_mode="floor").long(), (slots % case["page"]).long()
        for l in range(case["layers"]):
            _plain_write(s["k"][l], s["k_exp"][l], s["new"][l][0][keep], p, o)
            _plain_write(s["v"][l], s["v_exp"][l], s["new"][l][1][keep], p, o)
            out, lse = _plain_attn(s, l)
            outs.append(out)
        return outs + ([lse] if case["lse"] else []) + _state_out(s)
    return list(_plain_verify(s))


# ---------------------------------------------------------------- work
def work(case):
    """Bytes and operations of one pass; a domain's prompt is read once, not
    once a request."""
    kind = case["kind"]
    if kind in ("write", "read"):
        rows = 2 * case["tokens"] * case["heads"]
        return {"bytes": rows * (3 * case["dim"] + 1) + 4 * case["tokens"], "flops": 3 * rows * case["dim"]}
    if kind == "verify":
        # the row at which a request stops, of p and (for a rejected draft) q
        n, V = case["requests"], case["vocab"]
        rows = n * (2 if case["d_hi"] else 1)
        return {"bytes": rows * V * 4 + n * (8 + 12 * case["d_hi"]), "flops": 4 * rows * V}
    q_len, kv_len, group, group_len = _batch(case)
    H, KV, D, layers = case["heads"], case["kv_heads"], case["dim"], case.get("layers", 1)
    used = {g for g in group if g >= 0}
    tokens = sum(kv_len) + sum(group_len[g] for g in used)
    pairs = 0
    for q, kv, g in zip(q_len, kv_len, group):
        first = kv - q + 1  # own tokens that the first row sees
        pairs += sum(max(0, first + i) for i in range(q)) + (q * group_len[g] if g >= 0 else 0)
    b = tokens * KV * 2 * (D + 1) + 2 * sum(q_len) * H * D * 2 + (sum(q_len) * H * 4 if case["lse"] else 0)
    if kind == "step":
        b += sum(q_len) * KV * 2 * (3 * D + 1)
    return {"bytes": layers * b, "flops": layers * 4 * pairs * H * D}


# ---------------------------------------------------------------- 64 bits
def _exact_pow2(k):
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_rows(x):
    """The values the stored codes stand for in units of their power of two,
    and that power's exponent, from the definition."""
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
    return torch.round(y / step) * step, torch.where(a > 0, k, torch.full_like(k, -127.0)).squeeze(-1)


def _exact_cache(codes, exps):
    return codes.double() * torch.where(exps > 0, _exact_pow2(exps.long() - 127), 0.0).unsqueeze(-1)


def _exact_attn(s, host, layer, codes):
    """Request by request, head group by head group."""
    case = s["case"]
    P, H, KV, D = case["page"], case["heads"], case["kv_heads"], case["dim"]
    q_len, kv_len, own_ptr, own_pages, group, group_len, pre_ptr, pre_pages = host
    k, v = codes
    out = torch.zeros((sum(q_len), H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((sum(q_len), H), -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for b, n in enumerate(q_len):
        gl = group_len[group[b]] if group[b] >= 0 else 0
        lists = []
        if gl:
            lists.append((pre_pages[pre_ptr[group[b]]:pre_ptr[group[b] + 1]], gl))
        if kv_len[b]:
            lists.append((own_pages[own_ptr[b]:own_ptr[b + 1]], kv_len[b]))
        if lists:
            kk = torch.cat([k(layer, p).transpose(1, 2).reshape(-1, KV, D)[:m] for p, m in lists])
            vv = torch.cat([v(layer, p).transpose(1, 2).reshape(-1, KV, D)[:m] for p, m in lists])
            pos = torch.arange(len(kk), device="cuda")
            for i0 in range(0, n, 256):
                i = torch.arange(i0, min(n, i0 + 256), device="cuda")
                see = pos[None, :] <= (gl + kv_len[b] - n + i)[:, None]
                q = s["q"][layer][at + i].double().view(len(i), KV, H // KV, D)
                sc = torch.einsum("ikgd,lkd->kgil", q, kk) * s["scale"]
                sc = sc.masked_fill(~see, -math.inf)
                ls = torch.logsumexp(sc, -1)
                p = torch.exp(sc - torch.where(ls == -math.inf, 0.0, ls)[..., None])
                out[at + i] = torch.einsum("kgil,lkd->ikgd", p, vv).reshape(len(i), H, D)
                lse[at + i] = ls.permute(2, 0, 1).reshape(len(i), H)
        at += n
    return out, lse


def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None  # whole numbers
    s = prepare(case, seed)
    P = case["page"]
    if kind == "write":
        p, o = s["slots"].long() // P, s["slots"].long() % P
        k, v = s["k"][0].double(), s["v"][0].double()
        k[p, :, o] = _exact_rows(s["new_k"])[0]
        v[p, :, o] = _exact_rows(s["new_v"])[0]
        return [k[None], None, v[None], None]
    if kind == "read":
        p, o = s["slots"].long() // P, s["slots"].long() % P
        return [_exact_cache(s[x][0][p, :, o], s[x + "_exp"][0][p, :, o]) for x in ("k", "v")]
    pairs = sum(max(1, n) * m for n, m in zip([case["q_hi"]] * case["requests"], [case["own_hi"] + case["prompt"]] * case["requests"]))
    if case.get("layers", 1) * pairs * case["heads"] * case["dim"] * 4 > 6e12:
        return None
    if kind == "step":
        keep = (s["slots"] >= 0).nonzero().squeeze(1)
        p, o = s["slots"][keep].long() // P, s["slots"][keep].long() % P
        for l in range(case["layers"]):
            for x, rows in (("k", s["new"][l][0]), ("v", s["new"][l][1])):
                c, e = _exact_rows(rows[keep])
                s[x][l].view(torch.uint8)[p, :, o] = c.to(torch.float8_e4m3fn).view(torch.uint8)
                s[x + "_exp"][l][p, :, o] = (e + 127).to(torch.uint8)

    def rows(x):
        return lambda layer, pages: _exact_cache(s[x][layer][pages], s[x + "_exp"][layer][pages])
    outs, lse = [], None
    for l in range(case.get("layers", 1)):
        out, lse = _exact_attn(s, s["host"], l, (rows("k"), rows("v")))
        outs.append(out)
    res = outs + ([lse] if case["lse"] else [])
    if kind == "step":
        res += [s["k"].double(), None, s["v"].double(), None]
    return res
