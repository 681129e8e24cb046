"""GPU attention over the 4-bit cache against the 64-bit definition.

Tolerances (before any run): products of decoded keys and bfloat16 queries are
exact, their float32 sums over d <= 128 terms are off by at most
D = (d + 8) 2^-24 sum |q k| scale, plus the exponential's and scale's
2^-20 (1 + |s|) with |s| <= sum |q k| scale; the probabilities are rounded to
bfloat16 (2^-8 relative, half its spacing of 2^-7; once more for sums of any
length at 2^-15) and so is the output. With A = sum p |v| (>= |out|):
    |out - ref| <= 2^-8 |ref| + A (1.01 * 2^-8 + 2 D') + 1e-30
    |lse - ref| <= D' + 2^-18 + 2^-21 |ref|,   D' = D + 2^-20 (1 + sum |q k| scale).
"""
import random

import pytest
import torch

from oracle import serving_oracle as orc
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu
NEG_INF = float("-inf")


def _check(out, lse, ref):
    o, z, (absv, reach) = ref
    d = o.shape[-1]
    dd = (d + 8) * 2.0 ** -24 * reach + 2.0 ** -20 * (1 + reach)
    got, gz = out.cpu().double(), lse.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(o)) and torch.equal(torch.isnan(gz), torch.isnan(z))
    tol = 2.0 ** -8 * o.abs() + absv * (1.01 * 2.0 ** -8 + 2 * dd[..., None]) + 1e-30
    fine = ~torch.isnan(o)
    assert ((got - o).abs() <= tol)[fine].all(), float(((got - o).abs() / tol)[fine].max())
    assert torch.equal(gz == NEG_INF, z == NEG_INF)
    fine = torch.isfinite(z)
    tol = dd + 2.0 ** -18 + 2.0 ** -21 * z.abs()
    assert ((gz - z).abs() <= tol)[fine].all(), float(((gz - z).abs() / tol)[fine].max())


def _cache(total, page, hkv, d, seed, unused=255):
    """A cache for the given lengths on pages in random order; every slot that holds no key has NaN scales."""
    g = torch.Generator().manual_seed(seed)
    count = [(n + page - 1) // page for n in total]
    pages = sum(count) + 2
    order = torch.randperm(pages, generator=g).int()
    codes = torch.randint(0, 256, (pages, hkv, page, 2, d // 2), generator=g, dtype=torch.uint8)
    scales = torch.randint(122, 128, (pages, hkv, page, 2, d // 32), generator=g, dtype=torch.uint8)
    table = torch.full((len(total), max(count + [1]) + 1), -1, dtype=torch.int32)
    at, used = 0, torch.zeros(pages, page, dtype=torch.bool)
    for r, (n, c) in enumerate(zip(total, count)):
        own = order[at:at + c]
        table[r, :c] = own
        for i in range(n):
            used[own[i // page], i % page] = True
        at += c
    if unused is not None:
        scales[~used[:, None].expand(pages, hkv, page)] = unused
    return codes, scales, table


def _run(q, codes, scales, table, cu, seq, **kw):
    dev = {k: (v.cuda() if torch.is_tensor(v) else v) for k, v in kw.items()}
    return lt.cache4_attention(q.cuda(), codes.cuda(), scales.cuda(), table.cuda(),
                               torch.tensor(cu, dtype=torch.int32, device="cuda"),
                               torch.tensor(seq, dtype=torch.int32, device="cuda"), **dev)


def _both(total, new, hq, hkv, d, page, seed, extra=0, **kw):
    codes, scales, table = _cache(total, page, hkv, d, seed)
    g = torch.Generator().manual_seed(seed + 1)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    q = torch.randn(cu[-1] + extra, hq, d, generator=g).to(torch.bfloat16)
    scale = kw.pop("scale", d ** -0.5)
    print("attn4", total[:6], new[:6], hq, hkv, d, page, flush=True)
    out, lse = _run(q, codes, scales, table, cu, total, scale=scale, **kw)
    names = dict(visible_start="start", visible_end="end", selected="selected", selected_start="base")
    ref = orc.attention(q, codes, scales, table, cu, total, scale, **{names[k]: v for k, v in kw.items()})
    _check(out, lse, ref)
    return out, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 1), (8, 2), (16, 1), (20, 1), (34, 1), (64, 1), (70, 1)])
def test_decode_head_layouts(lib, hq, hkv, d):
    _both([1, 17, 300, 64], [1, 1, 1, 1], hq, hkv, d, 16, seed=hq + d)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 257, 1000, 5000])
def test_decode_lengths(lib, n):
    _both([n], [1], 8, 2, 128, 64, seed=n)


@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 256])
def test_page_sizes(lib, page):
    _both([700, 3, 90], [1, 2, 1], 4, 2, 64, page, seed=page)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("total,new,hq,hkv", [
    ([40, 7, 1, 300], [3, 7, 0, 5], 6, 2),
    ([200], [200], 4, 1),
    ([333, 64], [129, 64], 8, 2),
    ([500, 31, 260], [17, 31, 130], 16, 1),
    ([96], [65], 3, 3),
    ([1200, 5], [300, 1], 4, 2),
])
def test_several_tokens_a_request(lib, total, new, hq, hkv, d):
    _both(total, new, hq, hkv, d, 16, seed=sum(new) + d)


def test_many_requests(lib):
    rng = random.Random(4)
    total = [rng.choice([1, 2, 30, 33, 64, 150, 400]) for _ in range(200)]
    _both(total, [1] * 200, 8, 2, 64, 16, seed=9)
    new = [min(n, rng.choice([0, 1, 1, 4])) for n in total]
    _both(total, new, 8, 2, 64, 16, seed=10, extra=3)


def test_more_requests_than_a_wave_searches_at_once(lib):
    rng = random.Random(5)
    total = [rng.randint(1, 40) for _ in range(4100)]
    _both(total, [1 if rng.random() < 0.9 else 0 for _ in total], 2, 1, 64, 16, seed=11)


@pytest.mark.parametrize("total,new", [([300, 50, 9], [5, 2, 9]), ([600], [150]), ([300, 40], [1, 1])])
def test_visible_ranges_and_empty_rows(lib, total, new):
    g = torch.Generator().manual_seed(3)
    tokens = sum(new)
    start = torch.randint(-5, 200, (tokens,), generator=g, dtype=torch.int32)
    end = torch.randint(-5, 330, (tokens,), generator=g, dtype=torch.int32)
    end[0] = start[0].clamp(min=0)                 # a row that sees nothing
    if tokens > 3:
        start[2], end[2] = 0, 2**31 - 1            # everything
        start[3], end[3] = 2**31 - 1, 2**31 - 1
    _both(total, new, 8, 2, 128, 16, seed=21, visible_start=start, visible_end=end)
    _both(total, new, 8, 2, 64, 16, seed=22, visible_start=torch.minimum(start, end))
    _both(total, new, 8, 2, 64, 16, seed=23, visible_end=end)


def test_window(lib):
    total, new = [900, 30, 2000], [3, 30, 1]
    end = torch.tensor([n - q + i + 1 for n, q in zip(total, new) for i in range(q)], dtype=torch.int32)
    _both(total, new, 12, 4, 64, 16, seed=31, visible_start=(end - 100).clamp(min=0), visible_end=end)


def _lists(total, new, k, seed, pad=0.1):
    g = torch.Generator().manual_seed(seed)
    rows = []
    for n, q in zip(total, new):
        for i in range(q):
            e = n - q + i + 1
            p = torch.randperm(e, generator=g)[:k]
            p = torch.cat((p, torch.full((k - len(p),), -1)))
            p[torch.rand(k, generator=g) < pad] = -1
            rows.append(p)
    return torch.stack(rows).int()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k", [1, 31, 32, 100, 129, 512])
@pytest.mark.parametrize("hq,hkv", [(64, 1), (8, 2), (40, 1)])
def test_lists(lib, hq, hkv, k, d):
    total, new = [400, 5, 77], [2, 5, 1]
    _both(total, new, hq, hkv, d, 16, seed=k + hq, selected=_lists(total, new, k, seed=k))


def test_lists_with_entries_that_do_not_count(lib):
    total, new, k = [300, 90], [3, 2], 64
    sel = _lists(total, new, k, seed=1)
    sel[0] = -1                                     # nothing
    sel[1, ::2] = torch.arange(32, dtype=torch.int32) + 290     # partly beyond the visible end
    sel[2, :10] = sel[2, 10:20]                     # listed twice
    sel[3, 0], sel[3, 1], sel[3, 2] = 2**31 - 1, -2**31, 10**6
    _both(total, new, 8, 1, 128, 16, seed=41, selected=sel)
    start = torch.tensor([0, 10, 20, 5, 85], dtype=torch.int32)
    _both(total, new, 8, 1, 128, 16, seed=42, selected=sel, visible_start=start)
    # positions in an array that holds the sequences one after the other
    base = torch.tensor([100, 100, 100, 400, 400], dtype=torch.int32)
    packed = torch.where(sel >= 0, (sel.long() + base[:, None]).clamp(max=2**31 - 1).int(), sel)
    _both(total, new, 8, 1, 128, 16, seed=41, selected=packed, selected_start=base)
    wide = torch.full((5, 200), 7, dtype=torch.int32)
    wide[:, 50:114] = sel
    _both(total, new, 8, 1, 128, 16, seed=41, selected=wide.cuda()[:, 50:114].cpu())


def test_list_rows_with_a_stride(lib):
    total, new, k = [300, 90], [3, 2], 64
    sel = _lists(total, new, k, seed=2)
    wide = torch.full((5, 200), 7, dtype=torch.int32, device="cuda")
    wide[:, 50:114] = sel.cuda()
    codes, scales, table = _cache(total, 16, 1, 64, seed=2)
    q = torch.randn(5, 4, 64).to(torch.bfloat16)
    a = _run(q, codes, scales, table, [0, 3, 5], total, selected=sel)
    b = lt.cache4_attention(q.cuda(), codes.cuda(), scales.cuda(), table.cuda(),
                            torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda"),
                            torch.tensor(total, dtype=torch.int32, device="cuda"), selected=wide[:, 50:114])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_long_list_many_tokens(lib):
    total, new = [3000], [40]
    _both(total, new, 16, 1, 64, 64, seed=51, selected=_lists(total, new, 1500, seed=51, pad=0.0))


def test_whole_list_equals_dense(lib):
    total, new = [500, 64], [1, 1]
    codes, scales, table = _cache(total, 16, 2, 128, seed=61)
    q = torch.randn(2, 8, 128).to(torch.bfloat16)
    sel = torch.arange(500, dtype=torch.int32).expand(2, 500).contiguous()
    a = _run(q, codes, scales, table, [0, 1, 2], total)
    b = _run(q, codes, scales, table, [0, 1, 2], total, selected=sel)
    kv = [orc.attention(q, codes, scales, table, [0, 1, 2], total, 128 ** -0.5)]
    _check(*a, kv[0])
    _check(*b, kv[0])


def test_masked_values_that_are_not_finite_stay_out(lib):
    """Keys and values that a row does not see hold NaN; rows that see one are NaN where the definition is."""
    total, new, hkv, d, page = [200, 70], [6, 70], 2, 128, 16
    codes, scales, table = _cache(total, page, hkv, d, seed=71)
    for pos, what, blk in ((197, 1, 2), (198, 0, 1), (150, 1, 0), (199, 1, 3)):
        scales[table[0, pos // page], 1, pos % page, what, blk] = 255
    for pos, what, blk in ((40, 1, 1), (60, 0, 0)):
        scales[table[1, pos // page], 0, pos % page, what, blk] = 255
    g = torch.Generator().manual_seed(72)
    q = torch.randn(76, 8, d, generator=g).to(torch.bfloat16)
    cu = [0, 6, 76]
    out, lse = _run(q, codes, scales, table, cu, total)
    ref = orc.attention(q, codes, scales, table, cu, total, d ** -0.5)
    assert torch.isnan(ref[0]).any() and not torch.isnan(ref[0]).all()
    _check(out, lse, ref)
    start = torch.full((76,), 151, dtype=torch.int32)
    start[6:] = 0
    out, lse = _run(q, codes, scales, table, cu, total, visible_start=start)
    _check(out, lse, orc.attention(q, codes, scales, table, cu, total, d ** -0.5, start=start))
    sel = _lists(total, new, 40, seed=73)
    out, lse = _run(q, codes, scales, table, cu, total, selected=sel)
    _check(out, lse, orc.attention(q, codes, scales, table, cu, total, d ** -0.5, selected=sel))


def test_padded_batch_and_missing_pages(lib):
    total, new = [90, 40], [2, 1]
    out, lse = _both(total, new, 8, 2, 128, 16, seed=81, extra=5)
    assert (out[3:] == 0).all() and (lse[3:] == NEG_INF).all()
    sel = torch.cat((_lists(total, new, 20, seed=82), torch.zeros(5, 20, dtype=torch.int32)))
    codes, scales, table = _cache(total, 16, 2, 128, seed=83)
    table[0, 1], table[0, 3], table[1, 0] = -1, 10**6, -5     # keys on these pages do not count
    q = torch.randn(8, 8, 128).to(torch.bfloat16)
    cu = [0, 2, 3]
    ref = orc.attention(q, codes, scales, table, cu, total, 0.1)
    _check(*_run(q, codes, scales, table, cu, total, scale=0.1), ref)
    ref = orc.attention(q, codes, scales, table, cu, total, 0.1, selected=sel)
    _check(*_run(q, codes, scales, table, cu, total, scale=0.1, selected=sel), ref)


def test_no_requests_and_no_tokens(lib):
    codes, scales, table = _cache([16], 16, 1, 64, seed=1)
    i = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(3, 4, 64, device="cuda").to(torch.bfloat16)
    for sel in (None, torch.zeros(3, 5, **i)):
        out, lse = lt.cache4_attention(q, codes.cuda(), scales.cuda(), torch.empty(0, 1, **i), torch.zeros(1, **i),
                                       torch.empty(0, **i), selected=sel)
        assert (out == 0).all() and (lse == NEG_INF).all()
    out, lse = lt.cache4_attention(q[:0], codes.cuda(), scales.cuda(), table.cuda(), torch.zeros(2, **i),
                                   torch.tensor([16], **i))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 1.0, 30.0])
def test_scales_and_peaked_rows(lib, scale):
    _both([300, 20], [1, 5], 4, 1, 64, 16, seed=91, scale=scale)


def test_infinite_queries(lib):
    """+inf scores give NaN, as the definition does; a row of -inf scores has no weights and gives 0."""
    codes, scales, table = _cache([40], 16, 1, 64, seed=95)
    codes[..., 0, :] = 0x22                         # keys of ones
    q = torch.randn(2, 2, 64).to(torch.bfloat16)
    q[0, 0, 3], q[1, 1, 5] = float("inf"), NEG_INF
    out, lse = _run(q, codes, scales, table, [0, 2], [40])
    assert torch.isnan(out[0, 0]).all() and torch.isnan(lse[0, 0])
    assert (out[1, 1] == 0).all() and lse[1, 1] == NEG_INF
    assert torch.isfinite(out[0, 1]).all() and torch.isfinite(out[1, 0]).all()


def test_strided_queries_without_lse(lib):
    total, new = [120, 33], [1, 3]
    codes, scales, table = _cache(total, 16, 2, 64, seed=97)
    wide = torch.randn(4, 3 * 8 * 64).to(torch.bfloat16).cuda()
    q = wide[:, 512:1024].view(4, 8, 64)
    i = dict(dtype=torch.int32, device="cuda")
    args = (codes.cuda(), scales.cuda(), table.cuda(), torch.tensor([0, 1, 4], **i), torch.tensor(total, **i))
    a, none = lt.cache4_attention(q, *args, return_lse=False)
    assert none is None
    b, _ = lt.cache4_attention(q.contiguous(), *args)
    assert torch.equal(a, b)


def test_another_stream_and_repeated_calls(lib):
    total, new = [2000, 100], [1, 1]
    codes, scales, table = _cache(total, 64, 2, 128, seed=98)
    i = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(2, 16, 128).to(torch.bfloat16).cuda()
    args = (codes.cuda(), scales.cuda(), table.cuda(), torch.tensor([0, 1, 2], **i), torch.tensor(total, **i))
    a = lt.cache4_attention(q, *args)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = lt.cache4_attention(q, *args, stream=s)
    s.synchronize()
    c = lt.cache4_attention(q, *args)
    for x in (b, c):
        assert torch.equal(a[0], x[0]) and torch.equal(a[1], x[1])


def test_page_offsets_past_32_bits(lib):
    """Rows whose byte offset does not fit 32 bits: a cache of more than 4 GiB, keys on its last pages."""
    hkv, d, page = 8, 128, 64
    pages = (5 << 30) // (hkv * page * d)
    codes = torch.zeros(pages, hkv, page, 2, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.full((pages, hkv, page, 2, d // 32), 127, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(100, hkv, d, generator=g, device="cuda") for _ in range(2))
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    at = torch.arange(100, device="cuda")
    slots = table[0, at // page].long() * page + at % page
    lt.cache4_append(k, v, codes, scales, slots)
    q = torch.randn(1, 16, d, generator=g, device="cuda").to(torch.bfloat16)
    i = dict(dtype=torch.int32, device="cuda")
    out, lse = lt.cache4_attention(q, codes, scales, table, torch.tensor([0, 1], **i), torch.tensor([100], **i))
    own = torch.cat((codes[-1:], codes[:1])).cpu(), torch.cat((scales[-1:], scales[:1])).cpu()
    _check(out, lse, orc.attention(q.cpu(), *own, torch.tensor([[0, 1]]), [0, 1], [100], d ** -0.5))
    ks, vs = lt.cache4_read(codes, scales, slots)
    kv = orc.decode(*own)
    want = kv[at.cpu() // page, :, at.cpu() % page]
    assert torch.equal(ks.cpu().double(), want[:, :, 0]) and torch.equal(vs.cpu().double(), want[:, :, 1])


def test_argument_errors_raise(lib):
    codes, scales, table = (t.cuda() for t in _cache([16], 16, 1, 64, seed=1))
    i = dict(dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    cu, seq = torch.tensor([0, 1], **i), torch.tensor([16], **i)
    for bad in (dict(q=q.float()), dict(q=q[..., :32]), dict(cu=cu[:1]), dict(table=table.long()),
                dict(sel=torch.zeros(2, 3, **i)), dict(end=torch.zeros(2, **i)), dict(ws=torch.empty(8, **i)),
                dict(scale=0.0), dict(scales=scales[..., :1])):
        a = dict(dict(q=q, codes=codes, scales=scales, table=table, cu=cu, seq=seq, scale=1.0, sel=None, end=None,
                      ws=None), **bad)
        with pytest.raises(lt.LiteTopKError):
            lt.cache4_attention(a["q"], a["codes"], a["scales"], a["table"], a["cu"], a["seq"], a["scale"],
                                visible_end=a["end"], selected=a["sel"], workspace=a["ws"])


@pytest.mark.parametrize("reqs,new,hq,hkv,longest", [(2000, 1, 4, 2, 64), (300, 6, 8, 2, 80), (90, 40, 4, 1, 300),
                                                     (70, 3, 16, 4, 2500)])
def test_shares_of_several_tiles(lib, reqs, new, hq, hkv, longest):
    """More work than a share's smallest length for every block: shares hold whole tiles and parts of others."""
    rng = random.Random(reqs)
    total = [rng.choice([1, rng.randint(1, longest), longest]) for _ in range(reqs)]
    toks = [min(n, rng.choice([0, new, new])) for n in total]
    _both(total, toks, hq, hkv, 64, 16, seed=reqs)


def test_long_causal_prefill(lib):
    """Tiles from one key to the whole length: cuts by the tiles' own lengths."""
    _both([1500, 700], [1500, 700], 2, 1, 64, 64, seed=7)


def test_capture_in_a_graph(lib):
    """Every replay of a captured plan, append, attention and log probabilities equals the eager calls."""
    g = torch.Generator().manual_seed(1)
    i = dict(dtype=torch.int32, device="cuda")
    codes, scales = lt.cache4_empty(40, 16, 2, 64)
    table = torch.full((3, 8), -1, **i)
    free, used = torch.arange(39, -1, -1, **i), torch.zeros(1, **i)
    ctx, new = torch.zeros(3, **i), torch.tensor([30, 1, 17], **i)
    k, v, q = (torch.randn(48, h, 64, generator=g).cuda() for h in (2, 2, 8))
    q = q.to(torch.bfloat16)
    logits = torch.randn(48, 5000, generator=g).cuda()
    tok = torch.randint(0, 5000, (48,), generator=g).cuda()

    def step():
        p = lt.paged_plan(ctx, new, table, free, used, 16, 48)
        lt.cache4_append(k, v, codes, scales, p.slots)
        o, lse = lt.cache4_attention(q, codes, scales, table, p.cu_tokens, p.seq_lens)
        return [o, lse, *lt.token_logprobs(logits, tok, top=9), p.slots, p.status]

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(4):
        for t in got:
            t.zero_()
        codes.zero_()
        scales.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        step()                                     # the program's own eager work in between
        torch.cuda.synchronize()


@pytest.mark.parametrize("tokens,hq,hkv,d,k", [(280, 64, 1, 128, 97), (600, 40, 1, 64, 64), (520, 64, 1, 128, 130),
                                               (1030, 33, 1, 64, 1), (270, 100, 1, 128, 70), (130, 160, 2, 64, 129)])
def test_lists_of_many_tokens(lib, tokens, hq, hkv, d, k):
    """Wide tiles of one token each, with entries that do not count, empty lists and keys that are NaN."""
    total, new = [tokens - 23, 190], [tokens - 30, 30]
    sel = _lists(total, new, k, seed=k)
    sel[5] = -1
    sel[7, 0], sel[8, -1], sel[9, k // 2] = 2**31 - 1, -2**31, 10**6
    sel[10, :k // 2] = sel[10, k - k // 2:]         # listed twice
    codes, scales, table = _cache(total, 16, hkv, d, seed=k + 1)
    for r, pos, what, blk in ((0, 3, 1, 0), (0, 100, 1, 1), (1, 150, 0, 1), (1, 170, 1, d // 32 - 1)):
        scales[table[r, pos // 16], 0, pos % 16, what, blk] = 255
    table[0, 9] = -1                                # a page that is not there
    g = torch.Generator().manual_seed(tokens)
    q = torch.randn(tokens + 3, hq, d, generator=g).to(torch.bfloat16)
    sel = torch.cat((sel, torch.zeros(3, k, dtype=torch.int32)))
    cu = [0, tokens - 30, tokens]
    print("attn4 lists", tokens, hq, hkv, d, k, flush=True)
    out, lse = _run(q, codes, scales, table, cu, total, selected=sel)
    ref = orc.attention(q, codes, scales, table, cu, total, d ** -0.5, selected=sel)
    assert torch.isnan(ref[0]).any() and not torch.isnan(ref[0]).all()
    _check(out, lse, ref)
    assert (out[tokens:] == 0).all() and (lse[tokens:] == NEG_INF).all()


@pytest.mark.parametrize("hq,hkv,k", [(8, 2, 0), (64, 1, 0), (8, 2, 20), (64, 1, 20), (64, 1, 300)])
@pytest.mark.parametrize("lead", [1, 4, 300])
def test_tokens_before_the_first_request(lib, lead, hq, hkv, k):
    """cu_tokens that starts above 0: the tokens before it belong to no request, like those past its end."""
    total, new, tail = [90, 400, 7], [2, 40, 1], 3
    codes, scales, table = _cache(total, 16, hkv, 64, seed=lead)
    g = torch.Generator().manual_seed(lead + k)
    cu = [lead]
    for n in new:
        cu.append(cu[-1] + n)
    tokens = cu[-1] + tail
    q = torch.randn(tokens, hq, 64, generator=g).to(torch.bfloat16)
    kw = {}
    if k:
        sel = torch.zeros(tokens, k, dtype=torch.int32)
        sel[lead:cu[-1]] = _lists(total, new, k, seed=k)
        kw = dict(selected=sel)
    # memory that the results are likely to get: not zeros
    junk = [torch.full((tokens, hq, 64), 3.0, dtype=torch.bfloat16, device="cuda"),
            torch.full((tokens, hq), 5.0, device="cuda")]
    del junk
    print("attn4 lead", lead, hq, hkv, k, flush=True)
    out, lse = _run(q, codes, scales, table, cu, total, **kw)
    _check(out, lse, orc.attention(q, codes, scales, table, cu, total, 64 ** -0.5, **kw))
    for part in (slice(0, lead), slice(cu[-1], tokens)):
        assert (out[part] == 0).all() and (lse[part] == NEG_INF).all()
