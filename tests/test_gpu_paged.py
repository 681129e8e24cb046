"""GPU page plan and 4-bit pages against the plain definitions: whole numbers
and codes equal, values read back exact."""
import random

import pytest
import torch

from oracle import serving_oracle as orc
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu


def _plan(context, new, table, free, used, page, capacity):
    i = dict(dtype=torch.int32, device="cuda")
    t = torch.tensor(table, **i).reshape(len(context), -1)
    p = lt.paged_plan(torch.tensor(context, **i), torch.tensor(new, **i), t, torch.tensor(free, **i),
                      torch.tensor([used], **i), page, capacity)
    got = {n: getattr(p, n).tolist() for n in ("cu_tokens", "seq_lens", "slots", "positions", "free_used", "status")}
    return dict(got, table=t.tolist())


def _case(reqs, page, seed, width=9, new_hi=40, spare=1.0):
    rng = random.Random(seed)
    context = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, width * page)]) for _ in range(reqs)]
    new = [rng.choice([0, 1, 1, page, rng.randint(0, new_hi), -3]) for _ in range(reqs)]
    held = [-(-c // page) for c in context]
    need = sum(max(0, -(-(c + max(n, 0)) // page) - h) for c, n, h in zip(context, new, held))
    ids = list(range(sum(held) + need + 3))
    rng.shuffle(ids)
    at, table = 0, []
    for h in held:
        row = ids[at:at + h][:width]
        table.append(row + [-1] * (width - len(row)))
        at += h
    free = ids[at:]
    return context, new, table, free[:max(1, int(len(free) * spare))], sum(max(n, 0) for n in new)


@pytest.mark.parametrize("reqs", [1, 2, 63, 64, 65, 257, 1000])
@pytest.mark.parametrize("page,spare", [(1, 1.0), (16, 1.0), (16, 0.4), (64, 0.7)])
def test_plan_matches_definition(lib, reqs, page, spare):
    context, new, table, free, tokens = _case(reqs, page, seed=reqs * 7 + page, spare=spare)
    for used, capacity in ((0, tokens + 5), (min(2, len(free)), max(1, tokens // 2)), (len(free) + 4, tokens)):
        want = orc.paged_plan(context, new, table, free, used, page, capacity)
        assert _plan(context, new, table, free, used, page, capacity) == want


def test_plan_largest_request_count(lib):
    n = lt.LT_PLAN_MAX_REQUESTS
    context, new, table, free, tokens = _case(n, 16, seed=5, new_hi=3)
    assert _plan(context, new, table, free, 0, 16, tokens) == orc.paged_plan(context, new, table, free, 0, 16, tokens)


def test_plan_without_requests(lib):
    i = dict(dtype=torch.int32, device="cuda")
    p = lt.paged_plan(torch.empty(0, **i), torch.empty(0, **i), torch.empty(0, 4, **i), torch.arange(3, **i),
                      torch.tensor([2], **i), 16, 7)
    assert p.cu_tokens.tolist() == [0] and p.slots.tolist() == [-1] * 7 and p.free_used.tolist() == [2]


def test_plan_strided_table_and_sums_that_saturate(lib):
    i = dict(dtype=torch.int32, device="cuda")
    wide = torch.full((3, 40), -7, **i)
    table = wide[:, 4:12]
    p = lt.paged_plan(torch.tensor([0, 2**31 - 1, 5], **i), torch.tensor([20, 2**31 - 1, 2**31 - 1], **i), table,
                      torch.arange(100, 120, **i), torch.zeros(1, **i), 16, 64)
    assert p.status.tolist() == [0, 1, 1]
    assert p.cu_tokens.tolist() == [0, 20, 2**31 - 1, 2**31 - 1]
    assert p.slots[:20].tolist() == [1600 + j for j in range(16)] + [1616 + j for j in range(4)]
    assert p.slots[20:].tolist() == [-1] * 44
    assert table.tolist() == [[100, 101] + [-7] * 6, [-7] * 8, [-7] * 8]
    assert (wide[:, :4] == -7).all() and (wide[:, 12:] == -7).all()


def _inputs(rows, heads, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2, rows, heads, d, generator=g)
    x = x * torch.exp2(torch.randint(-12, 12, (2, rows, heads, d // 32, 1), generator=g).float()).expand(
        2, rows, heads, d // 32, 32).reshape(2, rows, heads, d)
    if rows > 2:
        x[0, 0, 0, :32] = 0.0
        x[0, 1, 0, :32] = torch.linspace(-7, 7, 32) + 0.25 * 0           # ties and the largest code
        x[1, 1, 0, :32] = torch.arange(32) * 0.25 - 3.75
        x[0, 2, 0, 5] = float("nan")
        x[1, 2, 0, 7] = float("-inf")
        x[1, 0, 0, :32] = 1.1754944e-38 * torch.arange(32).float()       # around the smallest exponents
        x[1, 0, 0, 32:64] = 1.4e-45 * torch.arange(32).float()           # denormal
        x[0, 2, 0, 32:64] = 3.0e38 * torch.linspace(-1, 1, 32)           # the largest
        x[0, 0, 0, 40] = 7.0                                             # exactly the bound of an exponent
        x[0, 1, 0, 32:64] = 0.0
        x[0, 1, 0, 33] = 7.0000005
    return x.to(dtype)


def _same(a, b):
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,heads,d,page", [(1, 1, 64, 1), (3, 1, 128, 16), (37, 3, 64, 8), (65, 8, 128, 64),
                                               (300, 2, 128, 4096)])
def test_append_and_read(lib, rows, heads, d, page, dtype):
    x = _inputs(rows, heads, d, dtype, seed=rows + d)
    pages = (rows + page - 1) // page + 1
    g = torch.Generator().manual_seed(rows)
    slots = torch.randperm(pages * page, generator=g)[:rows]
    codes, scales = lt.cache4_empty(pages, page, heads, d)
    codes.fill_(0xA5)
    scales.fill_(0x33)
    xd = x.cuda()
    lt.cache4_append(xd[0], xd[1], codes, scales, slots.cuda())
    k, v = lt.cache4_read(codes, scales, slots.cuda())
    for i, got in enumerate((k, v)):
        wc, ws = orc.quantise(x[i])
        own, off = slots // page, slots % page
        assert torch.equal(codes.cpu()[own, :, off, i], wc)
        assert torch.equal(scales.cpu()[own, :, off, i], ws)
        _same(got.cpu().double(), orc.decode(wc, ws))
    # nothing else is written
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[slots] = False
    c = codes.cpu().transpose(1, 2).reshape(pages * page, -1)[rest]
    s = scales.cpu().transpose(1, 2).reshape(pages * page, -1)[rest]
    assert (c == 0xA5).all() and (s == 0x33).all()


def test_slots_outside_the_cache_and_strided_rows(lib):
    heads, d, page, pages = 2, 128, 16, 3
    wide = torch.randn(6, 5 * heads * d, device="cuda")
    k = wide[:, heads * d:2 * heads * d].view(6, heads, d)
    v = wide[:, 3 * heads * d:4 * heads * d].view(6, heads, d)
    codes, scales = lt.cache4_empty(pages, page, heads, d)
    slots = torch.tensor([5, -1, pages * page, 47, 2**40, 0], device="cuda")
    lt.cache4_append(k, v, codes, scales, slots)
    a, b = lt.cache4_read(codes, scales, slots)
    for x, got in ((k, a), (v, b)):
        want = orc.decode(*orc.quantise(x.cpu()))
        for r, ok in enumerate([1, 0, 0, 1, 0, 1]):
            _same(got[r].cpu().double(), want[r] * ok)
    assert int((codes != 0).any(-1).any(-1).any(1).sum()) == 3


def test_all_codes_and_scales_read_exactly(lib):
    """Every code under every scale byte, those at the ends of bfloat16's range among them."""
    codes, scales = lt.cache4_empty(256, 1, 1, 64)
    codes[:, 0, 0, :, :8] = torch.arange(8, device="cuda", dtype=torch.uint8) * 34 + 16
    codes[:, 0, 0, :, 8:16] = torch.arange(8, 16, device="cuda", dtype=torch.uint8) * 17
    codes[:, 0, 0, :, 16:] = codes[:, 0, 0, :, :16]
    scales[:, 0, 0] = torch.arange(256, device="cuda", dtype=torch.uint8)[:, None, None]
    k, v = lt.cache4_read(codes, scales, torch.arange(256, device="cuda"))
    want = orc.decode(codes.cpu()[:, 0, 0], scales.cpu()[:, 0, 0]).to(torch.bfloat16)
    _same(k.cpu()[:, 0].double(), want[:, 0].double())
    _same(v.cpu()[:, 0].double(), want[:, 1].double())


def test_argument_errors_raise(lib):
    codes, scales = lt.cache4_empty(2, 16, 2, 128)
    k = torch.zeros(3, 2, 128, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(lt.LiteTopKError):
        lt.cache4_append(k, k, codes, scales, slots.int())
    with pytest.raises(lt.LiteTopKError):
        lt.cache4_append(k.half(), k.half(), codes, scales, slots)
    with pytest.raises(lt.LiteTopKError):
        lt.cache4_append(k[:, :1], k[:, :1], codes, scales, slots)
    with pytest.raises(lt.LiteTopKError):
        lt.cache4_read(codes, scales[:1], slots)
    with pytest.raises(lt.LiteTopKError):
        lt.cache4_append(k.transpose(0, 1).contiguous().transpose(0, 1), k, codes, scales, slots)


def test_results_on_another_stream_take_its_own_memory(lib):
    """Memory that was freed here while work queued here still reads it is not written by a call on another stream."""
    codes, scales = lt.cache4_empty(2, 16, 8, 128)
    slots = torch.zeros(1 << 14, dtype=torch.int64, device="cuda")
    zero = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(4)]
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    ones = torch.ones(4096, 4096, device="cuda")
    s = torch.cuda.Stream()
    for call in (lambda: lt.cache4_read(codes, scales, slots, stream=s),
                 lambda: [lt.paged_plan(zero[0], zero[1], table, zero[2], zero[3], 16, 1 << 22, stream=s).slots]):
        a = torch.arange(1 << 23, dtype=torch.int32, device="cuda")     # 32 MiB, as large as a result
        keep, want = torch.empty_like(a), a.cpu()
        torch.cuda.synchronize()
        x = ones
        for _ in range(20):
            x = torch.mm(x, ones)
        keep.copy_(a)
        lo, hi = a.data_ptr(), a.data_ptr() + a.numel() * 4
        del a
        for t in call():
            p = t.data_ptr()
            assert p + t.numel() * t.element_size() <= lo or p >= hi
        s.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(keep.cpu(), want)


def test_workspaces_that_are_not_memory_of_their_size(lib):
    """Host memory, and one byte that is expanded to a large size: neither is written."""
    codes, scales = lt.cache4_empty(2, 16, 1, 64)
    i = dict(dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    args = (q, codes, scales, torch.zeros(1, 2, **i), torch.tensor([0, 1], **i), torch.tensor([5], **i))
    x, tok = torch.zeros(2, 50000, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    for bad in (torch.empty(1 << 24, dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 24),
                torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(lt.LiteTopKError):
            lt.cache4_attention(*args, workspace=bad)
        with pytest.raises(lt.LiteTopKError):
            lt.token_logprobs(x, tok, top=5, workspace=bad)
    own = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    want = lt.cache4_attention(*args)
    assert all(torch.equal(a, b) for a, b in zip(lt.cache4_attention(*args, workspace=own), want))
    want = lt.token_logprobs(x, tok, top=5)
    assert all(torch.equal(a, b) for a, b in zip(lt.token_logprobs(x, tok, top=5, workspace=own), want))
