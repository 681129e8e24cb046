"""GPU: rotary positions (rotated, as fp8, and on the way into the 4-bit cache)
against the plain definition in 64 bits.

Rounding: sine and cosine are rounded to float32 (2^-24 relative; their 64-bit values
are better than 2^-35), then a product and a sum each (2^-24): of y = x1 c - x2 s at most
3 * 2^-24 of |x1 c| + |x2 s| <= amplitude * (|x1| + |x2|), and what comes after in their
products, below 2^-46. Written as bfloat16 half a step more (2^-8 of the value), as e4m3
2^-4 of the value or half the smallest step (2^-10 times the scale)."""
import math
from decimal import Decimal
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import serving_oracle as orc
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _freq(n, seed=0):
    return (10000.0 ** (-torch.arange(n, dtype=torch.float64) / max(n, 1)) * (1 + 0.01 * seed)).float()


def _x(tokens, heads, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(tokens, heads, d, generator=g) * (1 + 4 * torch.rand(d, generator=g))).to(TYPES[dtype])


def _pos(tokens, far, seed):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, far, (tokens,), generator=g).int()
    if tokens > 2:
        pos[0], pos[-1] = 0, -1
    return pos


def _limit(x, rot, n):
    """What float32 may be off by: 3 steps of |x1| + |x2| in the rotated part, nothing elsewhere."""
    a = x.double().abs()
    lim = torch.zeros_like(a)
    for i in range(n):
        u, v = ((rot.start + 2 * i, rot.start + 2 * i + 1) if rot.interleaved
                else (rot.start + i, rot.start + n + i))
        lim[..., u] = lim[..., v] = a[..., u] + a[..., v]
    return lim * (3.01 * STEP * abs(rot.amplitude))


def _check(got, x, pos, rot, inverse=False):
    n = rot.inv_freq.numel()
    want = orc.rotary(x, pos, rot.inv_freq.cpu(), rot.start, rot.interleaved, rot.amplitude, inverse)
    lim = _limit(x, rot, n)
    if got.dtype == torch.bfloat16:
        lim = lim * (1 + 2 ** -8) + 2.0 ** -8 * want.abs() + 1e-40
    assert torch.all((got.cpu().double() - want).abs() <= lim)


def _rot(n, start=0, interleaved=False, amplitude=1.0):
    return lt.Rotary(_freq(n).cuda(), start, interleaved, amplitude)


SHAPES = [  # tokens, heads, d, pairs, start: vectors of 8, 4, 2 and 1, whole heads and parts
    (1, 1, 128, 64, 0), (5, 3, 128, 32, 64), (3, 2, 64, 16, 16), (7, 8, 80, 20, 0), (4, 5, 80, 10, 2), (9, 1, 96, 48, 0),
    (2, 3, 6, 3, 0), (3, 1, 7, 2, 1), (2, 2, 1024, 512, 0), (2, 1, 1016, 100, 8), (3, 2, 1001, 77, 500), (5, 2, 192, 32, 128),
    (3, 2, 80, 27, 0), (5, 3, 80, 20, 40), (2, 2, 96, 12, 8), (2, 2, 64, 5, 2), (3, 1, 72, 36, 0), (2, 3, 40, 1, 36),
    (1, 64, 128, 64, 0), (130, 1, 128, 64, 0), (3, 2, 64, 0, 0), (2, 1, 1, 0, 0), (67, 40, 128, 64, 0), (33, 20, 256, 128, 0)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("types", ["f32-f32", "bf16-bf16", "f32-bf16"])
def test_rotary_matches_definition(lib, shape, interleaved, types):
    tokens, heads, d, n, start = shape
    a, b = types.split("-")
    x, pos, rot = _x(tokens, heads, d, a, 1), _pos(tokens, 131072, 2), _rot(n, start, interleaved, 1.25)
    got = lt.rotary(x.cuda(), pos.cuda(), rot, out_dtype=TYPES[b])
    assert got.dtype == TYPES[b] and got.shape == x.shape
    _check(got, x, pos, rot)
    if a == b:
        back = lt.rotary_backward(x.cuda(), pos.cuda(), rot)
        _check(back, x, pos, rot, inverse=True)


@pytest.mark.parametrize("far", [1 << 20, 0x7FFFFFFF])
def test_far_positions(lib, far):
    x, rot = _x(6, 2, 128, "f32", 3), _rot(64)
    pos = torch.tensor([far, far - 1, far // 3, 65537, 1, 0], dtype=torch.int64).clamp(max=0x7FFFFFFF).int()
    # 2^31 positions times a frequency of 1: the 64-bit angle itself is good to 2^31 * 2^-53 * (2 roundings)
    got = lt.rotary(x.cuda(), pos.cuda(), rot)
    want = orc.rotary(x, pos, rot.inv_freq.cpu())
    a = x.double().abs()
    both = torch.cat([a[..., :64] + a[..., 64:]] * 2, -1)
    assert torch.all((got.cpu().double() - want).abs() <= both * (3.01 * STEP + far * 2.0 ** -51))


@pytest.mark.parametrize("far", [1 << 20, 1 << 27, 0x7FFFFFFF])
@pytest.mark.parametrize("inverse", [False, True])
def test_far_angles_pair_by_pair(lib, far, inverse):
    """Against exact angles: pi / 2 as a 64-bit number is off by 2^-54 of itself, its quotient, the frequency's product
    and the position's by 2^-53 each, so an angle by 2^-51 of itself at most; c and s and the products as above."""
    pi = Fraction(Decimal("3.14159265358979323846264338327950288419716939937510582097494"))
    x, rot = _x(6, 2, 128, "f32", 4), _rot(64)
    pos = [far, far - 1, far - 12345, far // 3, 65537, 1]
    call = lt.rotary_backward if inverse else lt.rotary
    got = call(x.cuda(), torch.tensor(pos, dtype=torch.int32, device="cuda"), rot).cpu().double()
    for t, p in enumerate(pos):
        for i, f in enumerate(rot.inv_freq.tolist()):
            a = Fraction(f) * p
            r = float(a - 2 * pi * round(a / (2 * pi))) * (-1 if inverse else 1)
            u, v = x[t, :, i].double(), x[t, :, 64 + i].double()
            lim = (u.abs() + v.abs()) * (3.01 * STEP + float(a) * 2.0 ** -51)
            assert torch.all((got[t, :, i] - (u * math.cos(r) - v * math.sin(r))).abs() <= lim), (p, i)
            assert torch.all((got[t, :, 64 + i] - (v * math.cos(r) + u * math.sin(r))).abs() <= lim), (p, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 0), (1, 1), (0, 8)])
def test_slices_strides_and_in_place(lib, dtype, interleaved, pad, shift):
    tokens, heads, d, n = 21, 3, 64, 24
    whole = _x(tokens, 2 * heads + 1, d + pad + shift, dtype, 5).cuda()
    x = whole[:, heads:2 * heads, shift:shift + d]
    pos, rot = _pos(tokens, 5000, 6), _rot(n, 8, interleaved)
    got = lt.rotary(x, pos.cuda(), rot)
    _check(got, x.cpu(), pos, rot)
    # tokens inside heads
    turned = x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(lt.rotary(turned, pos.cuda(), rot), got)
    # into a slice, and in place: the values around stay
    place = torch.full_like(whole, 7.0)
    lt.rotary(x, pos.cuda(), rot, out=place[:, 1:1 + heads, shift:shift + d])
    assert torch.equal(place[:, 1:1 + heads, shift:shift + d], got)
    place[:, 1:1 + heads, shift:shift + d] = 7.0
    assert torch.all(place == 7.0)
    before = whole.clone()
    lt.rotary(x, pos.cuda(), rot, out=x)
    assert torch.equal(x, got)
    x.copy_(before[:, heads:2 * heads, shift:shift + d])
    assert torch.equal(whole, before)


def test_not_finite_stays_in_its_pair(lib):
    x = torch.ones(3, 1, 64)
    x[0, 0, 5], x[1, 0, 63], x[2, 0, 40] = math.nan, math.inf, math.nan
    y = lt.rotary(x.cuda(), torch.tensor([3, 4, -1], dtype=torch.int32, device="cuda"), _rot(16, 8)).cpu()
    bad = ~torch.isfinite(y)
    assert bad[0, 0].nonzero().flatten().tolist() == [5] and bad[1, 0].nonzero().flatten().tolist() == [63]
    assert torch.equal(y[2], torch.zeros(1, 64))
    y = lt.rotary(x.cuda(), torch.tensor([3, 4, 9], dtype=torch.int32, device="cuda"), _rot(32)).cpu()
    bad = ~torch.isfinite(y)
    assert [r[0].nonzero().flatten().tolist() for r in bad] == [[5, 37], [31, 63], [8, 40]]


def test_gradient_is_the_transpose(lib):
    """<rotary(x), g> = <x, rotary_backward(g)>, and differences along single values."""
    tokens, heads, d = 4, 2, 32
    x, g = _x(tokens, heads, d, "f32", 8), _x(tokens, heads, d, "f32", 9)
    pos, rot = _pos(tokens, 3000, 10), _rot(8, 4, amplitude=1.5)
    dx = lt.rotary_backward(g.cuda(), pos.cuda(), rot).cpu().double()
    y = lt.rotary(x.cuda(), pos.cuda(), rot).cpu().double()
    size = (x.double().abs().sum() * g.double().abs().max() * 1.5 * 2).item()
    assert abs((y * g.double()).sum() - (x.double() * dx).sum()) <= 6.1 * STEP * size
    for at in [(0, 0, 5), (1, 1, 13), (2, 0, 31), (3, 1, 7)]:
        z = x.clone()
        z[at] += 1.0
        change = (lt.rotary(z.cuda(), pos.cuda(), rot).cpu().double() - y) * g.double()
        # y is off by 3 steps of its pair on both sides
        slack = 2 * 3.01 * STEP * 1.5 * 2 * (x.abs().max() + 1).item() * g.abs().max().item() * 2 + 1e-6
        moved = z.double()[at] - x.double()[at]
        assert abs(change.sum() - dx[at] * moved) <= slack


def _decode_fp8(codes):
    c = codes.cpu().view(torch.uint8).to(torch.int32)
    sign, e, m = 1 - 2 * (c >> 7), (c >> 3) & 15, c & 7
    assert not torch.any((e == 15) & (m == 7))
    return sign * torch.where(e == 0, m.double() / 512, (1 + m.double() / 8) * torch.exp2(e.double() - 7))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fp8_matches_definition(lib, shape, interleaved, dtype):
    tokens, heads, d, n, start = shape
    x, pos, rot = _x(tokens, heads, d, dtype, 11), _pos(tokens, 131072, 12), _rot(n, start, interleaved)
    codes, scales = lt.rotary_fp8(x.cuda(), pos.cuda(), rot)
    want = orc.rotary(x, pos, rot.inv_freq.cpu(), start, interleaved)
    lim = _limit(x, rot, n)
    s = scales.cpu().double()
    assert torch.equal(torch.frexp(s)[0], torch.full_like(s, 0.5))
    top, off = want.abs().amax(-1), lim.amax(-1)
    assert torch.all(top <= 448 * s + off) and torch.all((top >= 224 * s - off) | (s == 2.0 ** -126))
    got = _decode_fp8(codes) * s[..., None]
    assert torch.all((got - want).abs() <= lim * (1 + 2 ** -4) + torch.maximum(2.0 ** -4 * want.abs(), s[..., None] * 2.0 ** -10))


def test_fp8_edges(lib):
    """Without a turn (position 0) codes and scales are exact functions of the row."""
    rows = torch.zeros(9, 1, 64)
    rows[0, 0, :4] = torch.tensor([448.0, -448.0, 1.0, 17.0])
    rows[1, 0, :4] = torch.tensor([np.nextafter(np.float32(448), np.float32(449)), 17.0, 19.0, -0.0])
    rows[3, 0, 0] = 1e-45
    rows[4, 0, 0], rows[5, 0, 0], rows[6, 0, 0] = math.inf, math.nan, -math.inf
    rows[7, 0, :2] = torch.tensor([3e38, -1.0])
    rows[8, 0, :8] = torch.tensor([448.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2 ** -9, 2.5 * 2 ** -9, 2.0 ** -10 * 1.001, 0.0, 1.0])
    codes, scales = lt.rotary_fp8(rows.cuda(), torch.zeros(9, dtype=torch.int32, device="cuda"), _rot(32))
    s = scales.flatten().cpu()
    want = [2.0 ** orc.fp8_exponent(float(r.abs().max())) if torch.isfinite(r).all() else math.nan for r in rows]
    assert np.array_equal(s.numpy(), np.array(want, np.float32), equal_nan=True)
    v = _decode_fp8(codes).reshape(9, 64)
    assert v[0, :4].tolist() == [448.0, -448.0, 1.0, 16.0] and v[1, :3].tolist() == [224.0, 8.0, 10.0]
    assert torch.all(v[4:7] == 0)
    assert v[8, :8].tolist() == [448.0, 2.0 ** -9, 0.0, 2.0 ** -8, 2.0 ** -8, 2.0 ** -9, 0.0, 1.0]


def test_fp8_feeds_the_indexer(lib):
    """Rotated queries and keys as fp8: the indexer's scores are those of the values they stand for."""
    nq, nk, h, d, k = 6, 700, 64, 128, 32
    q, key, rot = _x(nq, h, d, "bf16", 13), _x(nk, 1, d, "bf16", 14), _rot(32, 64, True)
    w = torch.rand(nq, h, generator=torch.Generator().manual_seed(15))
    qc, qs = lt.rotary_fp8(q.cuda(), torch.arange(nk - nq, nk, dtype=torch.int32, device="cuda"), rot)
    kc, ks = lt.rotary_fp8(key.cuda(), torch.arange(nk, dtype=torch.int32, device="cuda"), rot)
    idx, score = lt.indexer_topk(qc, w.cuda(), kc.view(nk, d), k, torch.arange(nk - nq + 1, nk + 1, dtype=torch.int32,
                                 device="cuda"), q_scale=qs, k_scale=ks.view(nk))
    qv = _decode_fp8(qc) * qs.cpu().double()[..., None]
    kv = (_decode_fp8(kc) * ks.cpu().double()[..., None])[:, 0]
    full = (torch.relu(torch.einsum("qhd,kd->qhk", qv, kv)) * w.double()[..., None]).sum(1)
    full = full.masked_fill(torch.arange(nk) > torch.arange(nk - nq, nk)[:, None], -math.inf)
    assert torch.allclose(score.cpu().double().sort(-1).values, full.topk(k).values.sort(-1).values, rtol=1e-4)


# ---- into the cache --------------------------------------------------------

def _append_case(rows, heads, d, dtype, page, hq=0, seed=20):
    k, v = _x(rows, heads, d, dtype, seed), _x(rows, heads, d, dtype, seed + 1)
    q = _x(rows, hq, d, dtype, seed + 2) if hq else None
    pages = (rows + page - 1) // page + 2
    g = torch.Generator().manual_seed(seed + 3)
    slots = torch.randperm(pages * page, generator=g)[:rows]
    return k, v, q, slots, lt.cache4_empty(pages, page, heads, d)


@pytest.mark.parametrize("rows,heads,d,page,n,start", [
    (1, 1, 128, 16, 64, 0), (64, 8, 128, 64, 64, 0), (77, 2, 64, 16, 32, 0), (50, 4, 128, 1, 32, 64), (33, 1, 64, 64, 8, 32),
    (40, 3, 128, 16, 20, 0), (21, 2, 64, 16, 5, 3), (31, 2, 128, 16, 36, 8), (26, 2, 64, 16, 12, 40), (17, 4, 128, 16, 39, 50), (9, 2, 128, 16, 0, 0), (300, 8, 64, 128, 16, 16), (18, 5, 128, 64, 63, 1)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_is_rotation_then_append(lib, rows, heads, d, page, n, start, interleaved, dtype):
    """Bit for bit what rotary in float32 and cache4_append make of the same rows (each of
    which is tested against its definition), and of the queries what rotary makes."""
    k, v, q, slots, (codes, scales) = _append_case(rows, heads, d, dtype, page, hq=2 * heads)
    pos, rot = _pos(rows, 1 << 20, 24), _rot(n, start, interleaved, 1.1)
    slots[rows // 2] = -1 if rows > 4 else slots[rows // 2]
    out = lt.cache4_append_rotary(k.cuda(), v.cuda(), codes, scales, slots.cuda(), pos.cuda(), rot, q=q.cuda())
    c2, s2 = lt.cache4_empty(codes.shape[0], page, heads, d)
    left = torch.where(pos < 0, torch.full_like(slots, -1), slots)
    lt.cache4_append(lt.rotary(k.cuda().float(), pos.cuda(), rot), v.cuda().float(), c2, s2, left.cuda())
    assert torch.equal(codes, c2) and torch.equal(scales, s2)
    assert torch.equal(out, lt.rotary(q.cuda(), pos.cuda(), rot, out_dtype=torch.bfloat16))
    c3, s3 = lt.cache4_empty(codes.shape[0], page, heads, d)
    assert lt.cache4_append_rotary(k.cuda(), v.cuda(), c3, s3, slots.cuda(), pos.cuda(), rot) is None
    assert torch.equal(codes, c3) and torch.equal(scales, s3)


@pytest.mark.parametrize("d,n", [(128, 64), (64, 16)])
def test_cached_keys_match_definition(lib, d, n):
    rows, heads, page = 70, 2, 16
    k, v, _, slots, (codes, scales) = _append_case(rows, heads, d, "bf16", page)
    pos, rot = _pos(rows, 131072, 25), _rot(n, d - 2 * n)
    lt.cache4_append_rotary(k.cuda(), v.cuda(), codes, scales, slots.cuda(), pos.cuda(), rot)
    got = lt.cache4_read(codes, scales, slots.cuda())[0].cpu().double().unflatten(-1, (-1, 32))
    want = orc.rotary(k, pos, rot.inv_freq.cpu(), d - 2 * n).unflatten(-1, (-1, 32))
    keep = pos >= 0
    off = _limit(k, rot, n).unflatten(-1, (-1, 32)).amax((-1), keepdim=True)
    top = want.abs().amax(-1, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2((top + off) / 7)))       # the larger one next to a border
    gap = torch.where(want.abs() < 2 * unit, 0.25, torch.where(want.abs() < 4 * unit, 0.5, 1.0)) * unit
    assert torch.all(((got - want).abs() <= gap + off)[keep])
    assert torch.all(got[~keep] == 0)


def test_append_slices_of_a_projection(lib):
    rows, hq, heads, d, page = 19, 8, 2, 128, 16
    whole = _x(rows, hq + 2 * heads, d, "bf16", 30).cuda()
    q, k, v = whole[:, :hq], whole[:, hq:hq + heads], whole[:, hq + heads:]
    pos, rot = _pos(rows, 4096, 31).cuda(), _rot(64)
    a, b = lt.cache4_empty(4, page, heads, d), lt.cache4_empty(4, page, heads, d)
    slots = torch.arange(rows, device="cuda")
    x = lt.cache4_append_rotary(k, v, *a, slots, pos, rot, q=q)
    y = lt.cache4_append_rotary(k.contiguous(), v.contiguous(), *b, slots, pos, rot, q=q.contiguous())
    assert torch.equal(x, y) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    # queries at an odd place: value by value
    flat = torch.zeros(rows * hq * d + 1, dtype=torch.bfloat16, device="cuda")
    flat[1:] = q.reshape(-1)
    z = lt.cache4_append_rotary(k, v, *a, slots, pos, rot, q=flat[1:].view(rows, hq, d))
    assert torch.equal(z, x) and torch.equal(a[0], b[0])


def test_values_that_are_not_finite(lib):
    k = torch.ones(2, 1, 64)
    k[0, 0, 3] = math.nan
    v = torch.ones(2, 1, 64)
    v[1, 0, 40] = math.inf
    c, s = lt.cache4_empty(1, 16, 1, 64)
    rot = _rot(16)          # pairs (i, i + 16) of the first block
    lt.cache4_append_rotary(k.cuda(), v.cuda(), c, s, torch.arange(2, device="cuda"),
                            torch.tensor([5, 6], dtype=torch.int32, device="cuda"), rot)
    kk, vv = (t.cpu().isnan().unflatten(-1, (2, 32)).all(-1) for t in lt.cache4_read(c, s, torch.arange(2, device="cuda")))
    assert kk[:, 0].tolist() == [[True, False], [False, False]] and vv[:, 0].tolist() == [[False, False], [False, True]]


def test_empty_calls(lib):
    rot = _rot(32)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    x = torch.zeros(0, 4, 64, device="cuda")
    assert lt.rotary(x, none, rot).shape == (0, 4, 64)
    codes, scales = lt.rotary_fp8(x, none, rot)
    assert codes.shape == (0, 4, 64) and scales.shape == (0, 4)
    c, s = lt.cache4_empty(2, 16, 4, 64)
    assert lt.cache4_append_rotary(x, x, c, s, none.long(), none, rot, q=x).shape == (0, 4, 64)
    assert lt.rotary(torch.zeros(3, 0, 64, device="cuda"), none.new_zeros(3), rot).shape == (3, 0, 64)


def test_argument_errors_raise(lib):
    rot, x = _rot(32), torch.zeros(3, 2, 64, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    c, s = lt.cache4_empty(2, 16, 2, 64)
    slots = torch.arange(3, device="cuda")
    calls = [
        lambda: lt.rotary(x.cpu(), pos, rot), lambda: lt.rotary(x, pos.cpu(), rot), lambda: lt.rotary(x, pos.long(), rot),
        lambda: lt.rotary(x, pos[:2], rot), lambda: lt.rotary(x.half(), pos, rot), lambda: lt.rotary(x[0], pos, rot),
        lambda: lt.rotary(x, pos, _rot(33)), lambda: lt.rotary(x, pos, _rot(16, 40)),
        lambda: lt.rotary(x, pos, lt.Rotary(rot.inv_freq.double())), lambda: lt.rotary(x, pos, lt.Rotary(rot.inv_freq.cpu())),
        lambda: lt.rotary(x, pos, rot, out=x[:2]), lambda: lt.rotary(x.bfloat16(), pos, rot, out_dtype=torch.float32),
        lambda: lt.rotary(x.transpose(1, 2), pos, lt.Rotary(rot.inv_freq[:1])),
        lambda: lt.rotary(x, pos, lt.Rotary(rot.inv_freq, amplitude=math.nan)),
        lambda: lt.rotary_fp8(x, pos, rot, out=(c, s)), lambda: lt.rotary_backward(x, pos[:1], rot),
        lambda: lt.cache4_append_rotary(x, x, c, s, slots, pos.long(), rot),
        lambda: lt.cache4_append_rotary(x, x, c, s, slots[:2], pos, rot),
        lambda: lt.cache4_append_rotary(x, x.bfloat16(), c, s, slots, pos, rot),
        lambda: lt.cache4_append_rotary(x, x, c, s, slots, pos, rot, q=x[:2]),
        lambda: lt.cache4_append_rotary(x, x, c, s, slots, pos, rot, q=x.bfloat16()),
        lambda: lt.cache4_append_rotary(x, x, c, s, slots.cpu(), pos, rot)]
    for i, call in enumerate(calls):
        with pytest.raises(lt.LiteTopKError):
            call()
            print("call %d was taken" % i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,n,start", [(64, 13, 0), (80, 27, 0), (64, 13, 9), (33, 9, 8), (1024, 505, 14), (1023, 501, 10),
                                       (17, 4, 0), (18, 8, 1), (40, 12, 16), (19, 5, 9)])
def test_parts_that_fill_no_vectors(lib, dtype, interleaved, d, n, start):
    """Vectors may cover the end of a length twice, in a result of its own: equal to the
    rotation in place, which covers it once, and to that of the same rows at an odd address."""
    tokens, heads = 37, 5
    x, pos, rot = _x(tokens, heads, d, dtype, 21).cuda(), _pos(tokens, 4000, 22), _rot(n, start, interleaved, 0.75)
    got = lt.rotary(x, pos.cuda(), rot)
    _check(got, x.cpu(), pos, rot)
    room = torch.full((tokens * heads * d + 3,), 7.0, dtype=x.dtype, device="cuda")
    odd = room[1:-2].view(tokens, heads, d)
    odd.copy_(x)
    assert torch.equal(lt.rotary(odd, pos.cuda(), rot), got)
    codes, scales = lt.rotary_fp8(x, pos.cuda(), rot)
    lt.rotary(odd, pos.cuda(), rot, out=odd)
    assert torch.equal(odd, got) and torch.all(room[:1] == 7.0) and torch.all(room[-2:] == 7.0)
    # fp8: half a step of the float32 rotation, whose own error is in _limit
    want = orc.rotary(x.cpu(), pos, rot.inv_freq.cpu(), rot.start, rot.interleaved, rot.amplitude, False)
    wide = scales.double().cpu()[..., None]
    err = (codes.cpu().view(torch.float8_e4m3fn).double() * wide - want).abs()
    lim = _limit(x.cpu(), rot, n) * (1 + 2 ** -4) + torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * wide)
    assert torch.all(err <= lim)
