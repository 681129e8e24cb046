"""GPU: beam selection against its definition in 64 bits.

A score is rounded once (2^-24 of its size). Its row's log sum comes from float32 terms:
a logit's distance to the lane's largest is rounded (2^-24), its exponent too (2^-24 of
itself) and the power of two (2^-23, one step); over the row the first two weigh no more
than the entropy, at most ln(vocab), so the sum's relative error, which is the log sum's
absolute one, stays below (2 ln(vocab) + 2 + 10) * 2^-24 with the ten additions of a
tile's chains. Order is exact where it does not hang on such errors: within a beam by
logit and token, and in what is returned by the returned scores."""
import math

import pytest
import torch

from oracle import serving_oracle as orc
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
INF = math.inf


def _check(logits, cum, top, scale=1.0, on_gpu=None):
    reqs, beams = cum.shape
    vocab = logits.shape[1]
    r = lt.beam_select(logits.cuda() if on_gpu is None else on_gpu, cum.cuda(), top, scale=scale)
    score, beam, token = (t.cpu() for t in r)
    assert score.shape == beam.shape == token.shape == (reqs, top)
    want = orc.beam_scores(logits, cum, scale)
    raw = logits.reshape(reqs, beams, vocab).double() + 0.0
    for b in range(reqs):
        flat = want[b].flatten()
        n = min(top, int((flat > -INF).sum()))
        assert torch.all(score[b, n:] == -INF) and torch.all(beam[b, n:] == -1) and torch.all(token[b, n:] == -1)
        if not n:
            continue
        s, w, v = score[b, :n].double(), beam[b, :n].long(), token[b, :n].long()
        assert int(w.min()) >= 0 and int(w.max()) < beams and int(v.min()) >= 0 and int(v.max()) < vocab
        x = raw[b, w, v]
        slack = (2 * math.log(max(vocab, 2)) + 12) * 2.0 ** -24
        tol = slack + 2.0 ** -24 * flat[flat > -INF].abs().max().item()
        assert torch.all((s - want[b, w, v]).abs() <= tol)
        # the returned order: score, beam, logit, token
        rows = list(zip((-s).tolist(), w.tolist(), (-x).tolist(), v.tolist()))
        assert rows == sorted(rows) and len({(p, q) for _, p, _, q in rows}) == n
        # of each beam its best, by logit and token
        for p in range(beams):
            mine = v[w == p]
            order = torch.sort(raw[b, p], descending=True, stable=True).indices
            assert torch.equal(mine, order[:mine.numel()])
        # nothing better is left out
        left = want[b].clone()
        left[w, v] = -INF
        assert left.max() <= s[-1] + tol or n < top
        if n < top:
            assert not torch.any(left > -INF)


def _draw(rows, vocab, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(rows, vocab, generator=g) * spread).to(TYPES[dtype])


def _cum(reqs, beams, seed):
    return -5 - 3 * torch.rand(reqs, beams, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("reqs,beams,vocab,top", [
    (1, 1, 1, 1), (2, 3, 1, 5), (3, 2, 7, 4), (1, 4, 32000, 8), (5, 5, 1001, 10), (2, 16, 5003, 32), (1, 64, 777, 64),
    (1, 2, 131072, 64), (3, 8, 8192, 16), (2, 4, 8193, 8), (40, 8, 2047, 16), (300, 4, 1500, 8), (1, 1, 200001, 2), (1, 200, 50, 64),
    (600, 4, 5000, 8), (2, 32, 20000, 64), (70, 16, 2048, 32)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matches_definition(lib, reqs, beams, vocab, top, dtype):
    _check(_draw(reqs * beams, vocab, dtype, 1), _cum(reqs, beams, 2), top)


@pytest.mark.parametrize("kind", ["rising", "falling", "constant", "two values", "zeros of both signs", "repeated beams",
                                  "one token", "few values"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_orders_and_ties(lib, kind, dtype):
    reqs, beams, vocab, top = 2, 4, 20011, 24
    g = torch.Generator().manual_seed(3)
    cum = _cum(reqs, beams, 4)
    x = torch.zeros(reqs * beams, vocab)
    if kind == "rising":
        x += torch.linspace(-9, 9, vocab)
    elif kind == "falling":
        x += torch.linspace(9, -9, vocab)
    elif kind == "constant":
        cum[:] = -3.0
    elif kind == "two values":
        x += (torch.rand(x.shape, generator=g) < 0.001) * 4.0
    elif kind == "zeros of both signs":
        x = torch.where(torch.rand(x.shape, generator=g) < 0.5, -0.0, 0.0)
    elif kind == "repeated beams":
        x[:] = torch.randn(vocab, generator=g)
        cum[:] = -1.0
    elif kind == "one token":
        x[:] = -INF
        x[:, 12345] = 2.0
    else:
        x = torch.randint(0, 40, x.shape, generator=g).float() / 4
    _check(x.to(TYPES[dtype]), cum, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [300, 30011])
def test_masks_and_beams_that_are_not_alive(lib, dtype, vocab):
    reqs, beams, top = 7, 4, 12
    x, cum = _draw(reqs * beams, vocab, dtype, 5), _cum(reqs, beams, 6)
    rows = x.view(reqs, beams, vocab)
    rows[0] = -INF                                     # nothing to choose from
    rows[1, 1:] = -INF
    rows[1, 0, 5:] = -INF                              # five candidates
    rows[2, 1] = torch.finfo(rows.dtype).min           # a mask of the type's lowest value: all alike
    rows[2, 2, 7:] = torch.finfo(rows.dtype).min
    rows[3, 0, 17] = math.nan
    rows[3, 1, 18] = INF
    cum[4, 1:] = -INF                                  # the first step
    rows[4, 1:] = math.nan
    cum[5] = -INF
    cum[6, 2] = math.nan
    rows[6, :, ::2] = -INF
    _check(x, cum, top)


def _alike(cum, n):
    """What n equal logits score, and how far off a float32 may be: the terms are 1, their sum exact, the logarithm
    a few 2^-52 of itself; then one rounding."""
    want = cum - math.log(n)
    return want, 2.0 ** -24 * abs(want) + 1e-13


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [7, 300, 30011])
@pytest.mark.parametrize("scale", [1.0, 0.7, 100.0])
def test_rows_of_the_lowest_values(lib, dtype, vocab, scale):
    """By hand: a row of one value gives every token cum - log(vocab), a mask's lowest value or any other,
    and so does what a row keeps of a mask that leaves n equal ones."""
    low = torch.finfo(TYPES[dtype]).min
    values = [low, -low, -1e30, 1e30, 1e15, -1e12, 0.0]
    top, beams = 6, 2
    x = torch.zeros(len(values), beams, vocab, dtype=TYPES[dtype])
    for r, v in enumerate(values):
        x[r, 0] = v
        x[r, 1], x[r, 1, 1:6] = low, max(v, -1e30)     # five equal ones above a mask
    cum = torch.tensor([[-3.0, -3.0 - 2 * math.log(vocab)]]).repeat(len(values), 1)
    r = lt.beam_select(x.view(-1, vocab).cuda(), cum.cuda(), top, scale=scale)
    want, tol = _alike(-3.0, vocab)
    n = min(top, vocab)
    assert torch.all((r.score[:, :n].cpu().double() - want).abs() <= tol)
    assert torch.all(r.beam[:, :n] == 0) and torch.equal(r.token[:, :n].cpu(), torch.arange(n).int().repeat(len(values), 1))
    # the second beam alone
    cum[:, 0], cum[:, 1] = -INF, -2.0
    r = lt.beam_select(x.view(-1, vocab).cuda(), cum.cuda(), 5, scale=scale)
    want, tol = _alike(-2.0, 5)
    assert torch.all((r.score.cpu().double() - want).abs() <= tol)
    assert torch.all(r.beam == 1) and torch.equal(r.token.cpu(), torch.arange(1, 6).int().repeat(len(values), 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_of_the_lowest_values_beside_others(lib, dtype):
    """It takes its place among its request's beams, not before them, and so does a row of one large value
    (in the second request)."""
    reqs, beams, vocab = 2, 4, 5003
    x, cum = _draw(reqs * beams, vocab, dtype, 21), torch.full((reqs, beams), -4.0)
    rows = x.view(reqs, beams, vocab)
    rows[:, 2] = torch.finfo(rows.dtype).min
    rows[1, 3] = 3e38
    r = lt.beam_select(x.cuda(), cum.cuda(), 1)
    assert torch.all(r.beam != 2) and r.beam[1, 0] != 3
    _check(x, cum, 40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["random", "rising", "falling", "equal"])
@pytest.mark.parametrize("rows,vocab,scale", [(8, 32000, 1.0), (512, 1001, 0.7), (3, 131072, 1.4), (600, 20011, 1.0)])
def test_log_sums(lib, dtype, kind, rows, vocab, scale):
    """The log sum's own error: the beam's score so far is minus its best log probability, so that the result
    lies near 0, where float32 resolves it. A term's distance and its exponent are rounded (2^-24 of the distance
    each; weighted over the row at most 2 H, H its entropy, and what rescaling adds to a term's distance makes up
    its distance to the row's largest), its power of two is off by 2^-23, and so is every factor that brings a
    sum to a larger maximum: at most one a tile of 1024 (bf16: 2048) logits and 40 in the joins; chains and
    their joining round ten times. Terms of equal logits are 1 and their sums exact."""
    x = _draw(rows, vocab, dtype, 31)
    if kind == "equal":
        x[:] = 3.0
    elif kind != "random":
        x = x.sort(-1, descending=kind == "falling").values
    logp = torch.log_softmax(x.double() * scale, -1)
    best = logp.amax(-1, keepdim=True)
    r = lt.beam_select(x.cuda(), (-best).float().cuda(), 1, scale=scale)
    off = (r.score.cpu().double() - ((-best).float().double() + best)).abs()
    p = logp.exp()
    entropy = -torch.special.xlogy(p, p).sum(-1, keepdim=True)
    moved = vocab // (2048 if dtype == "bf16" else 1024) + 40
    if kind == "equal":
        assert torch.all(off <= 1e-12)
    else:
        assert torch.all(off <= (2 * entropy + 2 * (1 + moved) + 10) * 1.01 * 2.0 ** -24)


def _upper(score):
    """The upper half of a score's float32 as it is ordered (no score is above 0)."""
    return -(score.float().view(torch.int32) & 0x7FFFFFFF) >> 16


@pytest.mark.parametrize("kind,reqs,beams,vocab,top,cum", [
    ("equal", 2, 16, 20011, 64, -3.0), ("equal", 1, 64, 5000, 64, -3.0), ("equal", 2, 200, 50, 64, -3.0),
    ("few", 2, 16, 9000, 64, -3.0), ("random", 2, 32, 20000, 64, -600.0), ("random", 1, 16, 128000, 64, -1000.0),
    ("random", 1, 100, 2000, 40, -5000.0), ("dead", 2, 100, 300, 50, -3.0), ("dead", 3, 64, 700, 64, -900.0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_joins_of_many(lib, kind, reqs, beams, vocab, top, cum, dtype):
    """More than 512 of the beams' best reach what the n-th best has in its upper 16 bits: equal scores, or
    different ones far from 0, where those bits tell them apart by 4 and more. The join takes them one by one."""
    x = _draw(reqs * beams, vocab, dtype, 41)
    if kind in ("equal", "dead"):
        x[:] = 1.5
    elif kind == "few":
        x = (x > 2.0).to(x.dtype)
    c = torch.full((reqs, beams), cum)
    if kind == "random":
        c -= 3 * torch.rand(reqs, beams, generator=torch.Generator().manual_seed(42))
    if kind == "dead":
        c[:, 3::5], c[0, 1] = -INF, math.nan
    y = orc.beam_scores(x, c)
    mine = y.topk(min(top, vocab), -1).values.flatten(1)
    mine = torch.where(mine > -INF, mine, -3e38)
    assert torch.all((_upper(mine) >= _upper(mine.topk(top, -1).values[:, -1:])).sum(-1) > 520)
    _check(x, c, top)


@pytest.mark.parametrize("dtype,pad,shift", [("bf16", 1, 0), ("bf16", 0, 3), ("f32", 5, 1), ("f32", 0, 0)])
def test_strided_and_unaligned_rows(lib, dtype, pad, shift):
    reqs, beams, vocab, top = 3, 3, 4999, 7
    whole = _draw(reqs * beams, vocab + pad + shift, dtype, 7)
    whole[:, :shift] = 50.0
    if pad:
        whole[:, vocab + shift:] = 50.0
    gpu = whole.cuda()[:, shift:shift + vocab]
    _check(whole[:, shift:shift + vocab].contiguous(), _cum(reqs, beams, 8), top, on_gpu=gpu)


@pytest.mark.parametrize("scale,spread", [(0.7, 3.0), (1.4, 3.0), (1e-6, 3.0), (100.0, 3.0), (1.0, 1e4), (1e-30, 1e30)])
def test_scales(lib, scale, spread):
    _check(_draw(12, 3001, "f32", 9, spread), _cum(3, 4, 10), 9, scale)


def test_empty_and_repeated(lib):
    r = lt.beam_select(torch.zeros(0, 100, device="cuda"), torch.zeros(0, 4, device="cuda"), 3)
    assert r.score.shape == (0, 3)
    r = lt.beam_select(torch.zeros(8, 0, device="cuda"), torch.zeros(2, 4, device="cuda"), 3)
    assert torch.all(r.score == -INF) and torch.all(r.beam == -1) and torch.all(r.token == -1)
    x, cum = _draw(64, 40000, "bf16", 11).cuda(), _cum(8, 8, 12).cuda()
    first = lt.beam_select(x, cum, 16)
    for _ in range(3):
        again = lt.beam_select(x, cum, 16)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_a_larger_workspace_serves(lib):
    big = torch.full((lt.lt_beam_select_workspace_size(lt.LT_BF16, 64, 8, 50000, 32),), 255, dtype=torch.uint8, device="cuda")
    for reqs, beams, vocab, top in [(64, 8, 50000, 32), (1, 8, 50000, 32), (3, 1, 12345, 5), (64, 2, 900, 1)]:
        x, cum = _draw(reqs * beams, vocab, "bf16", 13).cuda(), _cum(reqs, beams, 14).cuda()
        a, b = lt.beam_select(x, cum, top, workspace=big), lt.beam_select(x, cum, top)
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_agrees_with_token_logprobs(lib):
    """With one beam at 0 the continuations are the best alternatives of the row."""
    x = _draw(6, 33333, "bf16", 15).cuda()
    a = lt.beam_select(x, torch.zeros(6, 1, device="cuda"), 20)
    b = lt.token_logprobs(x, torch.zeros(6, dtype=torch.long, device="cuda"), top=20)
    assert torch.equal(a.token, b.top_index)
    assert torch.allclose(a.score, b.top_logprob, atol=4e-6)


def test_argument_errors_raise(lib):
    x, cum = torch.zeros(8, 50, device="cuda"), torch.zeros(2, 4, device="cuda")
    calls = [lambda: lt.beam_select(x.cpu(), cum, 3), lambda: lt.beam_select(x, cum.cpu(), 3),
             lambda: lt.beam_select(x.half(), cum, 3), lambda: lt.beam_select(x, cum.double(), 3),
             lambda: lt.beam_select(x, cum[:1], 3), lambda: lt.beam_select(x, cum.t(), 3), lambda: lt.beam_select(x[0], cum, 3),
             lambda: lt.beam_select(x.t(), cum, 3), lambda: lt.beam_select(x, cum, 0), lambda: lt.beam_select(x, cum, 65),
             lambda: lt.beam_select(x, cum, 3, scale=0.0), lambda: lt.beam_select(x, cum, 3, scale=math.nan),
             lambda: lt.beam_select(x, cum, 3, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda")),
             lambda: lt.beam_select(x, cum, 3, workspace=torch.zeros(1 << 20, dtype=torch.uint8))]
    for call in calls:
        with pytest.raises(lt.LiteTopKError):
            call()
