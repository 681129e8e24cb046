"""Plain CPU definitions of the serving operators, in 64 bits and loops over
requests (test infrastructure): the page plan, the 4-bit cache, attention over
it, and token log probabilities with their gradient."""
from __future__ import annotations

import math

import numpy as np
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


# ---- page plan -------------------------------------------------------------

def paged_plan(context, new, table, free, used, page, capacity):
    """Request by request; lists and a table (list of lists) in, a dict out."""
    table = [list(r) for r in table]
    width = len(table[0]) if table else 0
    used = min(max(used, 0), len(free))
    cu, seq, status, slots, positions = [0], [], [], [], []
    next_page = used
    closed = False  # a request ran out of pages: no page is handed out any more
    for r, (c, n) in enumerate(zip(context, new)):
        c, n = max(c, 0), max(n, 0)
        held, total = -(-c // page), -(-(c + n) // page)
        st = 0
        if n > 0 and total > width:
            st = 1
        elif n > 0 and total > held and (closed or next_page + total - held > len(free)):
            st = 2
            closed = True
        if st == 0 and n > 0:
            for i in range(held, total):
                table[r][i] = free[next_page]
                next_page += 1
        for p in range(c, c + n):
            own = table[r][p // page] if st == 0 else -1
            slots.append(own * page + p % page if own >= 0 else -1)
            positions.append(p)
        cu.append(cu[-1] + n)
        seq.append(c if st else c + n)
        status.append(st)
    pad = max(0, capacity - len(slots))
    return dict(cu_tokens=cu, seq_lens=seq, status=status, slots=(slots + [-1] * pad)[:capacity],
                positions=(positions + [-1] * pad)[:capacity], free_used=[next_page], table=table)


# ---- 4-bit cache -----------------------------------------------------------

def block_exponent(top: float) -> int:
    """The smallest e with top <= 7 * 2^e, within [-127, 125] (6 * 2^125 is finite)."""
    e = -127
    if top > 0:
        e = max(-127, math.frexp(top / 7)[1] - 2)
        while top > math.ldexp(7.0, e):
            e += 1
    return min(e, 125)


def quantise(x: torch.Tensor):
    """Rows of values -> (codes uint8 [..., d / 2], scales uint8 [..., d / 32]), value by value."""
    flat = x.double().reshape(-1, 32).numpy()
    codes = np.zeros(flat.shape, dtype=np.uint8)
    scales = np.zeros(flat.shape[0], dtype=np.uint8)
    for b, row in enumerate(flat):
        if not np.all(np.isfinite(row)):
            scales[b] = 255
            continue
        e = block_exponent(float(np.max(np.abs(row))))
        scales[b] = e + 127
        for i, v in enumerate(row):
            a = math.ldexp(abs(float(v)), -e)
            # nearest level; the even code where two are as near
            best = min(range(8), key=lambda c: (abs(a - LEVELS[c]), c & 1))
            codes[b, i] = best | (8 if math.copysign(1.0, float(v)) < 0 else 0)
    codes = codes.reshape(*x.shape[:-1], -1, 2)
    packed = codes[..., 0] | (codes[..., 1] << 4)
    return torch.from_numpy(packed), torch.from_numpy(scales.reshape(*x.shape[:-1], -1))


def decode(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    """What codes and scale bytes stand for, float64."""
    level = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)
    v = torch.stack((level[(codes & 15).long()], level[(codes >> 4).long()]), -1).flatten(-2)
    s = torch.ldexp(torch.ones(scales.shape, dtype=torch.float64), scales.int() - 127)
    s[scales == 255] = float("nan")
    return v * s.repeat_interleave(32, -1)


# ---- attention ---------------------------------------------------------------

def attention(q, codes, scales, table, cu, seq, scale, start=None, end=None, selected=None, base=None):
    """(out, lse, spread) in float64: per token and head over the visible keys
    only. `spread` = (sum p |v| per output, largest sum |q_i k_i| * scale per
    row), which the tests' tolerances are made of."""
    t_all, hq, d = q.shape
    pages, hkv, page = codes.shape[:3]
    group = hq // hkv
    kv = decode(codes, scales)                       # [pages, hkv, page, 2, d]
    out = torch.zeros(t_all, hq, d, dtype=torch.float64)
    lse = torch.full((t_all, hq), float("-inf"), dtype=torch.float64)
    absv = torch.zeros_like(out)
    reach = torch.zeros_like(lse)
    for r in range(len(seq)):
        n = cu[r + 1] - cu[r]
        for i in range(n):
            t = cu[r] + i
            length = max(int(seq[r]), 0)
            e = length - n + i + 1 if end is None else int(end[t])
            e = min(max(e, 0), length)
            s = min(max(int(start[t]) if start is not None else 0, 0), e)
            keys = list(range(s, e))
            if selected is not None:
                b = int(base[t]) if base is not None else 0
                keys = [int(j) - b for j in selected[t] if s <= int(j) - b < e]
            place = [(int(table[r][j // page]), j % page) for j in keys
                     if j // page < len(table[r]) and 0 <= int(table[r][j // page]) < pages]
            if not place:
                continue
            own, off = (torch.tensor(c) for c in zip(*place))
            for h in range(hq):
                k, v = kv[own, h // group, off, 0], kv[own, h // group, off, 1]
                w = (k @ q[t, h].double()) * scale
                z = torch.logsumexp(w, 0)
                p = torch.exp(w - z)
                out[t, h] = p @ v
                lse[t, h] = z
                absv[t, h] = p @ v.abs()
                reach[t, h] = (k.abs() @ q[t, h].double().abs()).max() * scale
    return out, lse, (absv, reach)


# ---- log probabilities ---------------------------------------------------------

def ordered(row: torch.Tensor):
    """Indices of a row by the library's total order: higher first, -0 = +0, NaN last, equal ones by index."""
    vals = row.double().tolist()
    return sorted(range(len(vals)), key=lambda i: (math.isnan(vals[i]), 0.0 if math.isnan(vals[i]) else -vals[i], i))


def _log_softmax(logits, scale):
    """(lse, log p), from the row's maximum: a row of the lowest values is like any other."""
    y = logits.double() * scale
    top = y.amax(-1, keepdim=True)
    none = top == float("-inf")
    far = y - torch.where(none, torch.zeros_like(top), top)
    z = torch.log(torch.exp(far).sum(-1, keepdim=True))
    logp = torch.where(none, torch.full_like(y, float("-inf")), far - z)
    return (top + torch.where(none, torch.zeros_like(z), z)).squeeze(-1), logp


def token_logprobs(logits, tokens, top, scale):
    rows, vocab = logits.shape
    if vocab:
        lse, logp = _log_softmax(logits, scale)
    else:
        lse = torch.full((rows,), float("-inf"), dtype=torch.float64)
        logp = logits.double()
    p = torch.exp(logp)
    entropy = -torch.special.xlogy(p, p).sum(-1)
    logprob = torch.zeros(rows, dtype=torch.float64)
    index = torch.full((rows, top), -1, dtype=torch.int64)
    best = torch.full((rows, top), float("-inf"), dtype=torch.float64)
    for r in range(rows):
        if 0 <= int(tokens[r]) < vocab:
            logprob[r] = logp[r, int(tokens[r])]
        if top:
            o = ordered(logits[r])[:top]
            index[r, :len(o)] = torch.tensor(o)
            best[r, :len(o)] = logp[r, o]
    return logprob, entropy, lse, index, best


def token_logprobs_backward(logits, tokens, scale, g_logprob, g_entropy):
    lse, logp = _log_softmax(logits, scale)
    none = (lse == float("-inf"))[:, None]
    p = torch.exp(logp)
    xlogx = torch.special.xlogy(p, p)
    entropy = -xlogx.sum(-1, keepdim=True)
    hit = torch.arange(p.shape[1]) == tokens[:, None]
    counts = hit.any(-1, keepdim=True)
    g = torch.zeros_like(p)
    if g_logprob is not None:
        g = g + g_logprob.double()[:, None] * (hit.double() - p) * counts
    if g_entropy is not None:
        g = g - g_entropy.double()[:, None] * (xlogx + p * entropy)
    return torch.where(none, torch.zeros_like(g), scale * g)
