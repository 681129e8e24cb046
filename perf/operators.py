"""Performance cases of the serving operators: page plan, 4-bit cache, attention
over it, token log probabilities.

A case is a dict of plain values. ``op`` names the operator:

plan      ``paged_plan``: block tables and slot maps of a step from the requests'
          lengths. ``reqs`` requests hold ``lo``..``hi`` tokens and add
          ``qlo``..``qhi`` new ones.
append    ``cache4_append`` of ``rows`` new tokens and ``cache4_read`` of the same
          slots: keys and values are quantised into the pages and come back as
          the values that the cache then stands for.
attn      ``cache4_attention``: the new tokens of each request attend to the
          request's cached keys (all visible ones, or with ``k`` > 0 the ones on
          each token's list, as the indexer returns them; ``window`` > 0 limits
          the reach of a token).
logprob   ``token_logprobs``: log probability of a given token, entropy and the
          ``top`` best alternatives of every row of logits; with ``train`` also
          ``token_logprobs_backward`` of the first two.

Request lengths are spread over their range on a logarithmic scale and depend on
the case alone; values depend on the seed.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda"
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # E2M1 magnitudes by code
BLOCK = 32                                         # values that share a scale
NEG_INF = float("-inf")

# what a drawn case may cost at most: the largest listed one of its kind
MAX_PAIRS = {"dense": 1.5e9, "list": 1.3e8}  # (query row, key) pairs of attention
MAX_CACHE = 1.2e7                           # cached rows (tokens x heads)
MAX_LOGITS = 2.6e8                          # elements
MAX_APPEND = 3.3e7                          # values of the keys (and as many of the values)


def _attn(name, reqs, qlo, qhi, lo, hi, hq, hkv, d, page, k=0, window=0, lens=1):
    c = dict(op="attn", reqs=reqs, qlo=qlo, qhi=qhi, lo=lo, hi=hi, hq=hq, hkv=hkv, d=d, page=page, k=k, window=window,
             lens=lens)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the plan of a decode step: one new token for each of 64 requests
        dict(name="plan_decode", op="plan", reqs=64, qlo=1, qhi=1, lo=512, hi=131072, page=64, lens=1),
        # a step of a large server: 4096 requests, decoding, prefilling or idle
        dict(name="plan_mixed", op="plan", reqs=4096, qlo=0, qhi=512, lo=1, hi=16384, page=16, lens=2),
        # the new keys and values of a decode step
        dict(name="append_decode", op="append", rows=64, hkv=8, d=128, dtype="bf16", page=64),
        # the keys and values of a long prefill chunk, an odd number of rows in float32
        dict(name="append_chunk", op="append", rows=16381, hkv=8, d=128, dtype="f32", page=64),
        # one request that decodes at a short context: latency
        _attn("attn_decode_one", 1, 1, 1, 4001, 4001, 32, 8, 128, 64),
        # a decode step of a batch of ragged contexts up to 128K
        _attn("attn_decode_batch", 48, 1, 1, 1024, 131072, 64, 8, 128, 64, lens=3),
        # drafted tokens are verified: a few tokens for each request, 64-wide heads, a sliding window
        _attn("attn_verify_window", 37, 0, 5, 1, 40000, 12, 4, 64, 16, window=4096, lens=4),
        # a decode step of sparse attention: 64 heads share the 2048 keys that the indexer selected at 128K context
        _attn("attn_list_decode", 32, 1, 1, 2049, 131072, 64, 1, 128, 64, k=2048, lens=5),
        # a prefill chunk of sparse attention at 128K context
        _attn("attn_list_chunk", 1, 1000, 1000, 131072, 131072, 64, 1, 128, 64, k=2048),
        # dense prefill chunks of two requests at middling contexts
        _attn("attn_prefill", 2, 1999, 2048, 9000, 20000, 32, 8, 128, 64, lens=6),
        # the log probabilities that a decode step returns with its tokens
        dict(name="logprob_decode", op="logprob", rows=8, vocab=131072, ld=131072, dtype="bf16", top=20, scale=1.0,
             train=False),
        # policy-gradient training: log probabilities and entropies of sampled tokens, and the logits' gradient
        dict(name="logprob_train", op="logprob", rows=2039, vocab=128001, ld=128064, dtype="bf16", top=1, scale=0.9,
             train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "decode", "decode", "verify", "list", "list", "prefill", "logprob", "logprob"])
    if op == "plan":
        return dict(op="plan", reqs=_log(rng, 1, 4096), qlo=rng.choice([0, 1]), qhi=_log(rng, 1, 512), lo=1,
                    hi=_log(rng, 64, 131072), page=rng.choice([16, 64, 128]), lens=rng.randrange(1 << 20))
    if op == "append":
        d, hkv = rng.choice([64, 128]), rng.choice([1, 2, 4, 8])
        return dict(op="append", rows=max(1, min(_log(rng, 1, 16384), int(MAX_APPEND / (2 * hkv * d)))), hkv=hkv, d=d,
                    dtype=rng.choice(["bf16", "f32"]), page=rng.choice([16, 64, 128]))
    if op == "logprob":
        vocab = _log(rng, 1000, 260000)
        train = rng.random() < 0.5
        return dict(op="logprob", rows=max(1, min(_log(rng, 1, 4096), int(MAX_LOGITS / vocab / 2))), vocab=vocab,
                    ld=vocab + rng.choice([0, 0, 1, 8, 64]), dtype=rng.choice(["bf16", "f32"]),
                    top=rng.choice([0, 1, 5, 20, 64]), scale=rng.choice([1.0, 1.0, 0.7, 1.4]), train=train)
    d, page = rng.choice([64, 128, 128]), rng.choice([16, 64, 128])
    seed = rng.randrange(1 << 20)
    if op == "decode":
        hkv, hi = rng.choice([1, 2, 4, 8]), _log(rng, 256, 131072)
        reqs = max(1, min(_log(rng, 1, 256), int(MAX_CACHE / (hkv * hi))))
        return _attn(None, reqs, 1, 1, max(1, hi // 64), hi, hkv * rng.choice([1, 4, 7, 8]), hkv, d, page, lens=seed)
    if op == "verify":
        hkv, hi = rng.choice([1, 2, 4]), _log(rng, 64, 65536)
        reqs = max(1, min(_log(rng, 1, 128), int(MAX_CACHE / 4 / (hkv * hi))))
        return _attn(None, reqs, 0, rng.choice([2, 3, 5, 8]), 1, hi, hkv * rng.choice([2, 3, 8, 16]), hkv, d, page,
                     window=rng.choice([0, 0, 512, 4096]), lens=seed)
    if op == "list":
        k, hkv, group = rng.choice([256, 1000, 2048]), rng.choice([1, 1, 2]), rng.choice([8, 16, 64])
        reqs, hi = rng.choice([1, 1, 5, 24]), _log(rng, 1024, 131072)
        tokens = max(reqs, min(_log(rng, 1, 1000), int(MAX_PAIRS["list"] / (k * hkv * group))))
        q = max(1, min(tokens // reqs, hi))
        return _attn(None, reqs, q, q, max(q, hi // 16), hi, hkv * group, hkv, d, page, k=k, lens=seed)
    hkv, hi = rng.choice([1, 2, 8]), _log(rng, 512, 32768)
    group = rng.choice([4, 8])
    q = max(16, min(_log(rng, 64, 4096), hi, int(MAX_PAIRS["dense"] / (hi * hkv * group))))
    reqs = max(1, min(rng.choice([1, 2, 7]), int(MAX_PAIRS["dense"] / (hi * hkv * group * q))))
    return _attn(None, reqs, max(1, q // 2), q, max(q, hi // 4), hi, hkv * group, hkv, d, page,
                 window=rng.choice([0, 0, 1024]), lens=seed)


# ---------------------------------------------------------------------------
# lengths and inputs
# ---------------------------------------------------------------------------

def _lengths(case):
    """(total length, new tokens) of every request; the new tokens are the last ones of the total."""
    rng = random.Random(case["lens"])
    total, new = [], []
    for _ in range(case["reqs"]):
        n = _log(rng, case["lo"], case["hi"])
        q = min(rng.randint(case["qlo"], case["qhi"]), n)
        total.append(n)
        new.append(q)
    return total, new


def _visible(case):
    """Per request the (first, last + 1) visible key of every new token."""
    out = []
    for n, q in zip(*_lengths(case)):
        ends = [n - q + i + 1 for i in range(q)]
        out.append([(max(0, e - case["window"]) if case["window"] else 0, e) for e in ends])
    return out


def _quantise(x):
    """Rows of values to (codes, scale bytes): per 32 values the smallest power of
    two 2^e with max|x| <= 7 * 2^e, values rounded to the nearest E2M1 number
    (halfway: the even code); byte e + 127."""
    b = x.float().unflatten(-1, (-1, BLOCK))
    top = b.abs().amax(-1, keepdim=True)
    mant, exp = torch.frexp(top)                 # top = mant * 2^exp, mant in [0.5, 1)
    e = exp - 3 + (mant > 0.875).int()
    e = torch.where(top > 0, e, torch.full_like(e, -127)).clamp(-127, 125)
    a = (b / torch.ldexp(torch.ones_like(top), e)).abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, edge in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (a > edge) if i % 2 == 0 else (a >= edge)
    good = torch.isfinite(top)
    code = torch.where(good, code | (torch.signbit(b).to(torch.uint8) << 3), torch.zeros_like(code))
    scale = torch.where(good, e + 127, torch.full_like(e, 255)).to(torch.uint8).squeeze(-1)
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4), scale


def _values(codes, scales):
    """What codes and scale bytes stand for, in float32."""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    v = torch.stack((level[(codes & 15).int()], level[(codes >> 4).int()]), -1).flatten(-2)
    s = torch.ldexp(torch.ones(scales.shape, device=codes.device), scales.int() - 127)
    s = torch.where(scales == 255, torch.full_like(s, float("nan")), s)
    return (v.unflatten(-1, (-1, BLOCK)) * s.unsqueeze(-1)).flatten(-2)


def _rand_kv(gen, shape, d):
    """Keys or values as attention meets them: a few wide channels, a common offset."""
    wide = 1.0 + 5.0 * (torch.rand(d, generator=gen, device=DEV) < 0.05)
    shift = 0.3 * torch.randn(d, generator=gen, device=DEV)
    return torch.randn(*shape, d, generator=gen, device=DEV) * wide + shift


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = SimpleNamespace(case=case)
    if case["op"] == "logprob":
        x = 2.5 * torch.randn(case["rows"], case["ld"], generator=gen, device=DEV)
        s.tokens = torch.randint(0, case["vocab"], (case["rows"],), generator=gen, device=DEV)
        x.scatter_(1, s.tokens[:, None], 9.0 + torch.randn(case["rows"], 1, generator=gen, device=DEV))
        # every eighth row is constrained: most of its vocabulary is masked out
        rule = torch.rand(case["vocab"], generator=gen, device=DEV) < 0.9
        x[::8, :case["vocab"]].masked_fill_(rule, NEG_INF)
        s.tokens[5::16] = -1                    # positions that do not count
        s.logits = x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)[:, :case["vocab"]]
        s.g_logprob = torch.randn(case["rows"], generator=gen, device=DEV) / case["rows"]
        s.g_entropy = torch.full((case["rows"],), -0.01 / case["rows"], device=DEV)
        return s
    if case["op"] == "append":
        rows, page = case["rows"], case["page"]
        pages = (rows + page - 1) // page + 3
        typ = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        s.k = _rand_kv(gen, (rows, case["hkv"]), case["d"]).to(typ)
        s.v = _rand_kv(gen, (rows, case["hkv"]), case["d"]).to(typ)
        s.codes = torch.zeros(pages, case["hkv"], page, 2, case["d"] // 2, dtype=torch.uint8, device=DEV)
        s.scales = torch.zeros(pages, case["hkv"], page, 2, case["d"] // BLOCK, dtype=torch.uint8, device=DEV)
        order = torch.randperm(pages, generator=gen, device=DEV)
        at = torch.arange(rows, device=DEV)
        s.slots = order[at // page] * page + at % page
        return s

    page = case["page"]
    s.total, s.new = _lengths(case)
    total = torch.tensor(s.total, dtype=torch.int32, device=DEV)
    new = torch.tensor(s.new, dtype=torch.int32, device=DEV)
    width = max((n + page - 1) // page for n in s.total) + 1
    if case["op"] == "plan":
        s.context, s.new_lens = total - new, new
        held = (s.context + page - 1) // page
        mine = held.long().cumsum(0)
        need = sum((n + page - 1) // page for n in s.total) + 8
        order = torch.randperm(need, generator=gen, device=DEV).int()
        col = torch.arange(width, device=DEV)
        at = ((mine - held)[:, None] + col).clamp(max=need - 1)
        s.table = torch.where(col < held[:, None], order[at], torch.full_like(order[at], -1))
        s.free = order.flip(0).contiguous()      # the pages that nobody holds come first
        s.taken = torch.zeros(1, dtype=torch.int32, device=DEV)
        s.capacity = (sum(s.new) + 255) // 256 * 256
        return s

    # a cache whose pages lie in any order; slots past a request's end hold no key
    hkv, d = case["hkv"], case["d"]
    count = [(n + page - 1) // page for n in s.total]
    pages = sum(count) + 2
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    first = torch.tensor([0] + count, device=DEV).cumsum(0)[:-1]
    col = torch.arange(width, device=DEV)
    own_page = col < torch.tensor(count, device=DEV)[:, None]
    at = (first[:, None] + col).clamp(max=pages - 1)
    s.table = torch.where(own_page, order[at], torch.full_like(order[at], -1))
    s.codes = torch.empty(pages, hkv, page, 2, d // 2, dtype=torch.uint8, device=DEV)
    s.scales = torch.empty(pages, hkv, page, 2, d // BLOCK, dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 27) // (hkv * page * 2 * d))
    for i in range(0, pages, step):
        n = min(step, pages - i)
        s.codes[i:i + n], s.scales[i:i + n] = _quantise(_rand_kv(gen, (n, hkv, page, 2), d))
    room = (total[:, None] - col * page).clamp(0, page)[own_page]
    unused = torch.arange(page, device=DEV) >= room[:, None]
    mine = s.table[own_page].long()
    s.scales[mine] = torch.where(unused[:, None, :, None, None], torch.full_like(s.scales[:1], 255), s.scales[mine])
    s.cu = torch.tensor([0] + s.new, device=DEV).cumsum(0).int()
    s.seq = total
    tokens = sum(s.new)
    s.q = torch.randn(tokens, case["hq"], d, generator=gen, device=DEV).to(torch.bfloat16)
    seen = [p for r in _visible(case) for p in r]
    span = torch.tensor(seen, dtype=torch.int32, device=DEV).reshape(-1, 2)
    s.start = span[:, 0].contiguous() if case["window"] else None
    s.end = span[:, 1].contiguous()
    s.picked = None
    if case["k"]:
        k, e = case["k"], span[:, 1:].long()
        j = torch.arange(k, device=DEV)
        u = torch.rand(tokens, k, generator=gen, device=DEV)
        room = (e // k).clamp(min=1)
        p = j * e // k + (u * room).long().clamp(max=room - 1)
        p = torch.where(e >= k, p, torch.where(j < e, j, torch.full_like(p, -1)))
        long = e >= k                            # short lists keep their padding at the end
        mixed = p[:, torch.randperm(k, generator=gen, device=DEV)]
        s.picked = torch.where(long, mixed, p).int()
    s.scale = d ** -0.5
    s.req = [r for r, n in enumerate(s.new) for _ in range(n)]
    s.req = torch.tensor(s.req, dtype=torch.int64, device=DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    case = s.case
    if own:
        return _run_own(s, case)
    return {"plan": _plan, "append": _append, "attn": _attention, "logprob": _logprob}[case["op"]](s, case)


def _run_own(s, case):
    from paper_2607_11976_amd import litetopk as lt
    if case["op"] == "plan":
        p = lt.paged_plan(s.context, s.new_lens, s.table, s.free, s.taken, case["page"], s.capacity)
        return [p.cu_tokens, p.seq_lens, p.slots, p.positions, s.table, p.free_used, p.status]
    if case["op"] == "append":
        lt.cache4_append(s.k, s.v, s.codes, s.scales, s.slots)
        return list(lt.cache4_read(s.codes, s.scales, s.slots))
    if case["op"] == "attn":
        return list(lt.cache4_attention(s.q, s.codes, s.scales, s.table, s.cu, s.seq, scale=s.scale,
                                        visible_start=s.start, visible_end=s.end, selected=s.picked))
    r = lt.token_logprobs(s.logits, s.tokens, top=case["top"], scale=case["scale"])
    out = [r.logprob, r.entropy, r.lse, r.top_index, r.top_logprob]
    if case["train"]:
        out.append(lt.token_logprobs_backward(s.logits, s.tokens, r.lse, r.entropy, s.g_logprob, s.g_entropy,
                                              scale=case["scale"]))
    return out


def _plan(s, case):
    page, width, free = case["page"], s.table.shape[1], s.free.numel()
    held = (s.context + page - 1) // page
    pages = (s.context + s.new_lens + page - 1) // page
    long = (pages > width) & (s.new_lens > 0)
    need = torch.where((s.new_lens > 0) & ~long, pages - held, torch.zeros_like(held))
    upto = need.cumsum(0)
    out = (need > 0) & (s.taken + upto > free)
    status = long.int() + 2 * out.int()
    good = status == 0
    col = torch.arange(width, device=DEV)
    fresh = good[:, None] & (col >= held[:, None]) & (col < (held + need)[:, None])
    at = s.taken + (upto - need)[:, None] + col - held[:, None]
    table = torch.where(fresh, s.free[at.clamp(0, free - 1)], s.table)
    cu = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEV), s.new_lens.cumsum(0)))
    row = torch.arange(s.capacity, device=DEV)
    req = (torch.searchsorted(cu, row, right=True) - 1).clamp(max=case["reqs"] - 1)
    real = row < cu[-1]
    pos = torch.where(real, s.context[req] + row - cu[req], torch.full_like(row, -1))
    own_page = table[req, (pos // page).clamp(0, width - 1)].long()
    slots = torch.where(real & good[req] & (own_page >= 0), own_page * page + pos % page, torch.full_like(row, -1))
    seq = torch.where(good, s.context + s.new_lens, s.context)
    used = (s.taken + torch.where(good, need, torch.zeros_like(need)).sum()).int()
    return [cu.int(), seq, slots, pos.int(), table, used, status]


def _append(s, case):
    page, at = s.slots // case["page"], s.slots % case["page"]
    for i, x in enumerate((s.k, s.v)):
        codes, scales = _quantise(x)
        s.codes[page, :, at, i] = codes
        s.scales[page, :, at, i] = scales
    return [_values(s.codes[page, :, at, i], s.scales[page, :, at, i]).to(torch.bfloat16) for i in (0, 1)]


def _softmax_v(score, seen, v):
    """(weights of the visible keys applied to v, log of the weights' sum)."""
    score = torch.where(seen, score, torch.full_like(score, NEG_INF))
    m = score.amax(-1, keepdim=True)
    m = torch.where(m == NEG_INF, torch.zeros_like(m), m)
    p = torch.exp(score - m)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(z > 0, z, torch.ones_like(z))
    return o, (m + torch.log(z)).squeeze(-1)


def _attention(s, case):
    page, hkv, d = case["page"], case["hkv"], case["d"]
    group, tokens = case["hq"] // hkv, s.q.shape[0]
    q = s.q.float().view(tokens, hkv, group, d) * s.scale
    start = torch.zeros_like(s.end) if s.start is None else s.start
    if case["k"]:
        pos = s.picked.long()
        seen = (pos >= start[:, None]) & (pos < s.end[:, None])
        at = pos.clamp(min=0)
        own_page, off = s.table[s.req[:, None], at // page].long(), at % page
        kv = _values(s.codes[own_page, :, off], s.scales[own_page, :, off])  # [tokens, k, hkv, 2, d]
        k, v = kv[..., 0, :].transpose(1, 2), kv[..., 1, :].transpose(1, 2)
        o, lse = _softmax_v(torch.matmul(q, k.transpose(-1, -2)), seen[:, None, None], v)
        return [o.reshape(tokens, case["hq"], d).to(torch.bfloat16), lse.reshape(tokens, case["hq"])]
    out = torch.empty(tokens, case["hq"], d, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(tokens, case["hq"], device=DEV)
    t = 0
    for r, (n, new) in enumerate(zip(s.total, s.new)):  # ragged: each request has its own number of keys
        if not new:
            continue
        mine = s.table[r, :(n + page - 1) // page].long()
        kv = _values(s.codes[mine], s.scales[mine])                       # [pages, hkv, page, 2, d]
        kv = kv.permute(3, 1, 0, 2, 4).reshape(2, hkv, -1, d)[:, :, :n]
        rows = slice(t, t + new)
        at = torch.arange(n, device=DEV)
        seen = (at >= start[rows, None]) & (at < s.end[rows, None])       # [new, n]
        qr = q[rows].permute(1, 2, 0, 3).reshape(hkv, group * new, d)
        score = torch.matmul(qr, kv[0].transpose(-1, -2))
        o, z = _softmax_v(score.view(hkv, group, new, n), seen, kv[1][:, None])
        out[rows] = o.permute(2, 0, 1, 3).reshape(new, case["hq"], d).to(torch.bfloat16)
        lse[rows] = z.permute(2, 0, 1).reshape(new, case["hq"])
        t += new
    return [out, lse]


def _logprob(s, case):
    x = s.logits.float() * case["scale"]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == NEG_INF, torch.zeros_like(m), m))
    z = e.sum(-1, keepdim=True)
    lse = m + torch.log(torch.where(z > 0, z, torch.ones_like(z)))
    p = e / torch.where(z > 0, z, torch.ones_like(z))
    logp = x - lse
    logp = torch.where(x == NEG_INF, x, logp)
    plogp = torch.where(x == NEG_INF, torch.zeros_like(x), p * logp)
    entropy = -plogp.sum(-1)
    counts = (s.tokens >= 0) & (s.tokens < case["vocab"])
    tok = s.tokens.clamp(0, case["vocab"] - 1)[:, None]
    logprob = torch.where(counts, logp.gather(1, tok)[:, 0], torch.zeros_like(entropy))
    # larger first, equal ones by their index: one whole number holds both
    raw = s.logits.float() + 0.0
    bits = raw.view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) + (1 << 20) - 1 \
        - torch.arange(case["vocab"], device=DEV)
    top = min(case["top"], case["vocab"])
    index = (1 << 20) - 1 - (torch.topk(key, top, -1).values & ((1 << 20) - 1))
    out = [logprob, entropy, lse[:, 0], index.int(), logp.gather(1, index)]
    if case["train"]:
        g = -s.g_logprob[:, None] * counts[:, None] * p
        g.scatter_add_(1, tok, (s.g_logprob * counts)[:, None])
        g -= s.g_entropy[:, None] * (plogp + p * entropy[:, None])
        out.append((g * case["scale"]).to(s.logits.dtype))
    return out


# ---------------------------------------------------------------------------
# work and definition
# ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "plan":
        total, new = _lengths(case)
        page = case["page"]
        fresh = sum((n + page - 1) // page - (n - q + page - 1) // page for n, q in zip(total, new))
        return {"bytes": 8 * len(total) + 12 * len(total) + 8 * fresh + 12 * ((sum(new) + 255) // 256 * 256),
                "flops": 0}
    if case["op"] == "append":
        values = 2 * case["rows"] * case["hkv"] * case["d"]
        size = 2 if case["dtype"] == "bf16" else 4
        packed = values // 2 + values // BLOCK
        return {"bytes": values * size + packed + values * 2, "flops": 0}
    if case["op"] == "attn":
        pairs = rows = tokens = 0
        for spans in _visible(case):
            counts = [min(e - a, case["k"]) if case["k"] else e - a for a, e in spans]
            reach = max((e for _, e in spans), default=0) - min((a for a, _ in spans), default=0)
            pairs += sum(counts)
            rows += min(sum(counts), reach) if case["k"] else reach
            tokens += len(spans)
        row = case["hkv"] * (case["d"] + case["d"] // 16)
        return {"bytes": rows * row + tokens * case["hq"] * (4 * case["d"] + 4) + tokens * (4 * case["k"] + 8),
                "flops": 4 * case["d"] * pairs * case["hq"]}
    n, size = case["rows"] * case["vocab"], 2 if case["dtype"] == "bf16" else 4
    once = n * size + case["rows"] * (20 + 8 * case["top"])
    return {"bytes": once + (2 * n * size + 24 * case["rows"] if case["train"] else 0),
            "flops": n * (12 if case["train"] else 6)}


def exact(case, seed):
    if case["op"] == "plan":                  # whole numbers only
        return None
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attention, "logprob": _exact_logprob}[case["op"]](s, case)


def _exact_append(s, case):
    """The nearest level of every value under its block's power of two, by distance."""
    level = torch.tensor([LEVELS[i] for i in (0, 2, 4, 6, 1, 3, 5, 7)], dtype=torch.float64, device=DEV)
    out = []
    for x in (s.k, s.v):
        b = x.double().unflatten(-1, (-1, BLOCK))
        top = b.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top / 7)).clamp(-127, 125)
        e = torch.where((top > 7 * torch.exp2(e)) & (e < 125), e + 1, e)
        e = torch.where((top <= 7 * torch.exp2(e - 1)) & (e > -127), e - 1, e)
        unit = torch.exp2(e)
        a = (b / unit).abs()
        best, far = torch.zeros_like(a), torch.full_like(a, math.inf)
        for v in level:                       # even codes first: they win where two are as near
            near = (a - v).abs()
            best = torch.where(near < far, v.expand_as(a), best)
            far = torch.minimum(near, far)
        out.append((torch.copysign(best, b) * unit).flatten(-2))
    return out


def _decoded(codes, scales):
    """Codes and scale bytes in 64 bits, from the bit fields."""
    c = torch.stack((codes % 16, codes // 16), -1).flatten(-2).int()
    sign, e, m = 1 - 2 * (c // 8), (c // 2) % 4, c % 2
    v = torch.where(e == 0, 0.5 * m.double(), (1 + 0.5 * m.double()) * torch.exp2(e.double() - 1)) * sign
    return v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)


def _exact_attention(s, case):
    page, hq, d = case["page"], case["hq"], case["d"]
    group = hq // case["hkv"]
    out = torch.zeros(s.q.shape[0], hq, d, dtype=torch.float64, device=DEV)
    lse = torch.full((s.q.shape[0], hq), NEG_INF, dtype=torch.float64, device=DEV)
    t = 0
    for r, spans in enumerate(_visible(case)):
        at = torch.arange(s.total[r], device=DEV)
        pages = s.table[r].long()
        for i0 in range(0, len(spans), 256):
            part = spans[i0:i0 + 256]
            rows = slice(t + i0, t + i0 + len(part))
            for h in range(case["hkv"]):
                if case["k"]:
                    for j, (a, e) in enumerate(part):
                        pos = s.picked[t + i0 + j].long()
                        pos = pos[(pos >= a) & (pos < e)]
                        place = (pages[pos // page], h, pos % page)
                        kv = _decoded(s.codes[place], s.scales[place])
                        w = s.q[t + i0 + j, h * group:(h + 1) * group].double() @ kv[:, 0].T * s.scale
                        z = torch.logsumexp(w, -1)
                        lse[t + i0 + j, h * group:(h + 1) * group] = z
                        out[t + i0 + j, h * group:(h + 1) * group] = torch.exp(w - z[:, None]) @ kv[:, 1]
                    continue
                place = (pages[at // page], h, at % page)
                kv = _decoded(s.codes[place], s.scales[place])
                ab = torch.tensor(part, device=DEV)
                hide = (at < ab[:, :1]) | (at >= ab[:, 1:])
                for g in range(h * group, (h + 1) * group):
                    w = (s.q[rows, g].double() @ kv[:, 0].T * s.scale).masked_fill(hide, NEG_INF)
                    z = torch.logsumexp(w, -1)
                    lse[rows, g] = z
                    out[rows, g] = torch.exp(w - z[:, None]).masked_fill(hide, 0.0) @ kv[:, 1]
        t += len(spans)
    return [out, lse]


def _exact_logprob(s, case):
    parts = []
    for r in range(0, case["rows"], 128):
        x = s.logits[r:r + 128].double() * case["scale"]
        lse = torch.logsumexp(x, -1)
        logp = x - lse[:, None]
        p = torch.exp(logp)
        xlogx = torch.special.xlogy(p, p)
        entropy = -xlogx.sum(-1)
        tok = s.tokens[r:r + 128]
        hit = torch.arange(case["vocab"], device=DEV) == tok[:, None]
        logprob = torch.where(hit, logp, torch.zeros_like(logp)).sum(-1)
        part = [logprob, entropy, lse, torch.topk(logp, min(case["top"], case["vocab"]), -1).values]
        if case["train"]:
            g = s.g_logprob[r:r + 128].double()[:, None] * (hit.double() - p * hit.any(-1, keepdim=True))
            g = g - s.g_entropy[r:r + 128].double()[:, None] * (xlogx + p * entropy[:, None])
            part.append(case["scale"] * g)
        parts.append(part)
    whole = [torch.cat(c) for c in zip(*parts)]
    return whole[:3] + [None] + whole[3:]
