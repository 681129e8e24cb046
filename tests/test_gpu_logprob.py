"""GPU token log probabilities and their gradient against the 64-bit definition.

Tolerances (before any run): a scaled logit in powers of two is off by at most
d = 2^-22 Y + 2^-20, Y = the largest |y| log2 e of the row's finite entries
(float32 products, the running reference and the exponential's error), sums of
positive terms by 2^-20 relative. So
    lse: d;  log probabilities: 2 d;  entropy: 4 d (1 + H);
    gradient: r |g| + s (|g_lp| 4 d p + |g_H| 4 d p (1 + |log p| + H)) + 1e-30, r = 2^-8
    (bfloat16: half its spacing of 2^-7) or 2^-22 (float32).
"""
import math

import pytest
import torch

from oracle import serving_oracle as orc
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu
NEG_INF = float("-inf")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _slack(x, scale):
    y = torch.where(torch.isfinite(x.double()), x.double() * scale, torch.zeros(1, dtype=torch.float64))
    return 2.0 ** -22 * y.abs().amax(-1) * math.log2(math.e) + 2.0 ** -20


def _near(got, want, tol):
    got, want = got.cpu().double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    off = ((got - want).abs() / tol.expand_as(want))[fine]
    assert off.numel() == 0 or float(off.max()) <= 1.0, float(off.max())


def _both(x, tok, top, scale=1.0, x_dev=None):
    xd = x.cuda() if x_dev is None else x_dev
    print("logprob", tuple(x.shape), x.dtype, top, flush=True)
    r = lt.token_logprobs(xd, tok.cuda(), top=top, scale=scale)
    lp, h, lse, index, best = orc.token_logprobs(x, tok, min(top, x.shape[1]), scale)
    d = _slack(x, scale) if x.shape[1] else torch.ones(x.shape[0], dtype=torch.float64)
    _near(r.lse, lse, d)
    _near(r.logprob, lp, 2 * d)
    _near(r.entropy, h, 4 * d * (1 + h.nan_to_num()))
    assert torch.equal(r.top_index.cpu().long(), index)
    _near(r.top_logprob, best, 2 * d[:, None])
    return r


def _draw(rows, vocab, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (spread * torch.randn(rows, vocab, generator=g)).to(dtype)
    tok = torch.randint(0, max(vocab, 1), (rows,), generator=g)
    tok[::7] = -1
    if rows > 1:
        tok[1] = vocab          # outside
    return x, tok


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("rows,vocab", [(1, 1), (2, 7), (3, 8), (5, 63), (4, 64), (3, 1000), (2, 2049), (1, 50257),
                                        (9, 4097), (1100, 257), (1030, 9001)])
@pytest.mark.parametrize("top", [0, 1, 20, 64])
def test_matches_definition(lib, rows, vocab, dtype, top):
    if rows > 1000 and top not in (0, 20):
        top = 5
    x, tok = _draw(rows, vocab, dtype, seed=rows * 31 + vocab)
    if rows > 1000 and vocab > 1000:
        x, tok = x[:1030], tok
    _both(x, tok, top)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "two", "steps", "late"])
@pytest.mark.parametrize("rows", [1, 1024])
def test_orders_and_ties(lib, rows, kind, dtype):
    vocab = 20000 if rows == 1 else 9001
    i = torch.arange(vocab, dtype=torch.float32)
    x = {"rising": i * 0.01, "falling": -i * 0.01, "equal": torch.full((vocab,), 1.5), "two": (i % 2) * 3.0,
         "steps": torch.floor(i / 1000), "late": torch.where(i >= vocab - 70, 9.0, 0.0)}[kind].to(dtype)
    few = x[None].contiguous()
    tok = torch.tensor([vocab - 3])
    if rows == 1:
        _both(few, tok, 64)
        return
    many = few.expand(rows, vocab).contiguous().cuda()
    r = lt.token_logprobs(many, tok.expand(rows).contiguous().cuda(), top=64)
    lp, h, lse, index, best = orc.token_logprobs(few, tok, 64, 1.0)
    assert torch.equal(r.top_index.cpu().long(), index.expand(rows, 64))
    d = _slack(few, 1.0)
    _near(r.lse, lse.expand(rows), d)
    _near(r.logprob, lp.expand(rows), 2 * d)
    _near(r.entropy, h.expand(rows), 4 * d * (1 + h))


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
def test_masked_rows(lib, dtype):
    x, tok = _draw(8, 3001, dtype, seed=3)
    x[0] = NEG_INF                                   # nothing left
    x[1, :3000] = NEG_INF                            # one entry
    x[2, 5:] = NEG_INF
    x[3] = torch.finfo(dtype).min                    # the type's lowest value, not a mask: uniform
    x[4, ::2] = torch.finfo(dtype).min
    x[5, tok[5]] = NEG_INF
    tok[:3] = torch.tensor([2, 3000, 4])
    tok[0] = 17
    r = _both(x, tok, 20)
    assert r.lse[0] == NEG_INF and r.entropy[0] == 0 and r.logprob[0] == NEG_INF
    assert r.entropy[1] == 0 and r.logprob[1] == 0


def test_not_finite(lib):
    for n in (300, 20000):
        x = torch.randn(5, n)
        x[0, 7] = float("nan")
        x[1, 9] = float("inf")
        x[2, :] = float("nan")
        x[3, 11:] = float("nan")
        r = lt.token_logprobs(x.cuda(), torch.tensor([1, 2, 3, 4, 5]).cuda(), top=15)
        for row in (0, 1, 2, 3):
            assert torch.isnan(r.lse[row]) and torch.isnan(r.entropy[row]) and torch.isnan(r.logprob[row])
            assert r.top_index[row].tolist() == orc.ordered(x[row])[:15]
        assert torch.isfinite(r.lse[4])


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("pad,shift", [(1, 0), (5, 3), (64, 0), (7, 1)])
def test_strided_and_unaligned_rows(lib, dtype, pad, shift):
    x, tok = _draw(7, 5003, dtype, seed=pad)
    wide = torch.full((7, 5003 + pad + shift), 99.0, dtype=dtype, device="cuda")
    view = wide[:, shift:shift + 5003]
    view.copy_(x)
    r = _both(x, tok, 10, x_dev=view)
    g, td = torch.randn(7).cuda(), tok.cuda()
    a = lt.token_logprobs_backward(view, td, r.lse, r.entropy, g, None)
    b = lt.token_logprobs_backward(view.contiguous(), td, r.lse, r.entropy, g, None)
    assert torch.equal(a, b)
    # a gradient of unaligned rows, and nothing outside it
    out = torch.full((7, 5003 + pad + shift), 5.0, dtype=dtype, device="cuda")
    o = out[:, shift:shift + 5003]
    st = lt.lt_token_logprobs_backward(view.data_ptr(), lt._dtype_code(view), view.stride(0), 7, 5003,
                                       td.data_ptr(), 1.0, r.lse.data_ptr(), r.entropy.data_ptr(),
                                       g.data_ptr(), None, o.data_ptr(), out.stride(0),
                                       torch.cuda.current_stream().cuda_stream)
    assert st == lt.LT_OK and torch.equal(o, a)
    assert (out[:, :shift] == 5).all() and (out[:, shift + 5003:] == 5).all()


@pytest.mark.parametrize("scale", [0.05, 0.7, 1.0, 3.0])
@pytest.mark.parametrize("spread", [0.01, 3.0, 40.0])
def test_scales(lib, scale, spread):
    x, tok = _draw(6, 4001, torch.float32, seed=5, spread=spread)
    _both(x, tok, 5, scale=scale)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 9), (4, 1000), (2, 30011), (300, 515)])
@pytest.mark.parametrize("which", ["both", "logprob", "entropy", "none"])
def test_gradient_matches_formula(lib, rows, vocab, dtype, which):
    x, tok = _draw(rows, vocab, dtype, seed=rows + vocab)
    if rows > 2:
        x[2, : vocab // 2] = NEG_INF
    if rows > 3:
        x[3] = NEG_INF
    g = torch.Generator().manual_seed(8)
    gl = torch.randn(rows, generator=g) if which in ("both", "logprob") else None
    gh = torch.randn(rows, generator=g) if which in ("both", "entropy") else None
    scale = 0.8
    r = lt.token_logprobs(x.cuda(), tok.cuda(), scale=scale)
    got = lt.token_logprobs_backward(x.cuda(), tok.cuda(), r.lse, r.entropy, None if gl is None else gl.cuda(),
                                     None if gh is None else gh.cuda(), scale=scale)
    assert got.dtype == dtype and got.shape == x.shape
    want = orc.token_logprobs_backward(x, tok, scale, gl, gh)
    lse = torch.logsumexp(x.double() * scale, -1, keepdim=True)
    logp = torch.where(lse == NEG_INF, torch.full((1,), NEG_INF, dtype=torch.float64), x.double() * scale - lse)
    p = torch.exp(logp)
    far = torch.where(p > 0, logp.abs(), torch.zeros_like(p))
    h = orc.token_logprobs(x, tok, 0, scale)[1][:, None]
    d = _slack(x, scale)[:, None]
    tol = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22) * want.abs() + 1e-30
    if gl is not None:
        tol = tol + scale * gl.double().abs()[:, None] * 4 * d * p
    if gh is not None:
        tol = tol + scale * gh.double().abs()[:, None] * 4 * d * p * (1 + far + h)
    _near(got, want, tol)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
def test_gradient_of_rows_at_the_lowest_value(lib, dtype):
    """Every logit at the type's lowest value: a uniform row, its gradient g (1[tok] - 1/n)."""
    n = 3001
    x = torch.full((2, n), torch.finfo(dtype).min).to(dtype)
    x[1] = 5000.0
    tok = torch.tensor([7, 3000])
    r = lt.token_logprobs(x.cuda(), tok.cuda(), top=2)
    assert torch.allclose(r.entropy.cpu(), torch.full((2,), math.log(n)), rtol=1e-5)
    assert torch.allclose(r.logprob.cpu(), torch.full((2,), -math.log(n)), rtol=1e-5)
    g = torch.tensor([2.0, -3.0])
    got = lt.token_logprobs_backward(x.cuda(), tok.cuda(), r.lse, r.entropy, g.cuda(), None).cpu().double()
    want = orc.token_logprobs_backward(x, tok, 1.0, g, None)
    tol = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20) * want.abs()
    assert ((got - want).abs() <= tol).all()


def test_gradient_against_differences(lib):
    """Directional derivatives of the definition's sum g_lp lp + g_H H, by central differences in 64 bits."""
    x, tok = _draw(5, 700, torch.float32, seed=12)
    g = torch.Generator().manual_seed(13)
    gl, gh = torch.randn(5, generator=g), torch.randn(5, generator=g)
    r = lt.token_logprobs(x.cuda(), tok.cuda(), scale=1.3)
    grad = lt.token_logprobs_backward(x.cuda(), tok.cuda(), r.lse, r.entropy, gl.cuda(), gh.cuda(), scale=1.3).cpu()
    for s in range(5):
        v = torch.randn(5, 700, generator=g, dtype=torch.float64)

        def value(y):
            lp, h = orc.token_logprobs(y, tok, 0, 1.3)[:2]
            return float((gl.double() * lp + gh.double() * h).sum())

        want = (value(x.double() + 1e-5 * v) - value(x.double() - 1e-5 * v)) / 2e-5
        # the gradient's entries are off by 4 d of their terms: 1e-4 of the sums of magnitudes
        assert abs(float((grad.double() * v).sum()) - want) <= 1e-4 * float((grad.double() * v).abs().sum()) + 1e-6


def test_empty_and_repeated(lib):
    r = lt.token_logprobs(torch.empty(0, 50, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), top=3)
    assert r.logprob.shape == (0,) and r.top_index.shape == (0, 3)
    r = lt.token_logprobs(torch.empty(2, 0, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), top=3)
    assert r.lse.tolist() == [NEG_INF] * 2 and r.logprob.tolist() == [0.0, 0.0]
    x, tok = _draw(3, 90000, torch.bfloat16, seed=2)
    a = lt.token_logprobs(x.cuda(), tok.cuda(), top=30)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    xd, td = x.cuda(), tok.cuda()
    torch.cuda.synchronize()
    b = lt.token_logprobs(xd, td, top=30, stream=s)
    s.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_argument_errors_raise(lib):
    x = torch.zeros(3, 10, device="cuda")
    tok = torch.zeros(3, dtype=torch.int64, device="cuda")
    for args in ((x.half(), tok), (x, tok.int()), (x, tok[:2]), (x.t(), torch.zeros(10, dtype=torch.int64).cuda())):
        with pytest.raises(lt.LiteTopKError):
            lt.token_logprobs(*args)
    with pytest.raises(lt.LiteTopKError):
        lt.token_logprobs(x, tok, top=65)
    with pytest.raises(lt.LiteTopKError):
        lt.token_logprobs(x, tok, scale=0.0)
    with pytest.raises(lt.LiteTopKError):
        lt.token_logprobs_backward(x, tok, x[0], x[1])


def _gradient_and_formula(x, tok, scale, gl, gh):
    """(the kernel's gradient, the formula's, log p, the entropy) of both gradients, in 64 bits on the CPU."""
    xd, td = x.cuda(), tok.cuda()
    print("gradient", tuple(x.shape), x.dtype, scale, flush=True)
    r = lt.token_logprobs(xd, td, scale=scale)
    got = lt.token_logprobs_backward(xd, td, r.lse, r.entropy, None if gl is None else gl.cuda(),
                                     None if gh is None else gh.cuda(), scale=scale).cpu().double()
    y = x.double() * scale
    logp = y - y.amax(-1, keepdim=True)
    logp = logp - torch.logsumexp(logp, -1, keepdim=True)
    return got, orc.token_logprobs_backward(x, tok, scale, gl, gh), logp, -torch.special.xlogy(
        torch.exp(logp), torch.exp(logp)).sum(-1, keepdim=True)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("rows,vocab", [(1, 1), (6, 700), (5, 30011), (300, 515), (70, 4097)])
@pytest.mark.parametrize("which", ["both", "logprob", "entropy"])
def test_gradient_does_not_depend_on_an_offset(lib, rows, vocab, dtype, which):
    """Rows moved by up to thousands, next to rows that are not. The distance to a logit near the row's
    largest is exact to 2^-24, so p is off by at most e = 2^-20 + 2^-22 (8 + |log p|) relative (three
    roundings of log p's size, the exponential, a sum of positive terms), whatever the offset."""
    x, tok = _draw(rows, vocab, torch.float32, seed=rows + 3 * vocab)
    shift = torch.tensor([300.0, 0.0, -700.0, 2000.0, 120.0, -65.0])[torch.arange(rows) % 6]
    x = (x + shift[:, None]).to(dtype)
    g = torch.Generator().manual_seed(9)
    gl = torch.randn(rows, generator=g) if which != "entropy" else None
    gh = torch.randn(rows, generator=g) if which != "logprob" else None
    got, want, logp, h = _gradient_and_formula(x, tok, 1.0, gl, gh)
    p, far = torch.exp(logp), logp.abs()
    e = 2.0 ** -20 + 2.0 ** -22 * (8 + far)
    tol = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22) * want.abs() + 1e-30
    if gl is not None:
        tol = tol + gl.double().abs()[:, None] * e * p
    if gh is not None:
        tol = tol + gh.double().abs()[:, None] * 4 * e * p * (1 + far + h)
    _near(got, want, tol)
    if dtype == torch.float32 and which == "logprob":
        # g (1 - sum p): the sums' 2^-20 and the entries' own rounding
        assert (got.sum(-1).abs() <= 2.0 ** -19 * gl.double().abs()).all()


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("rows", [3, 130])
def test_gradient_at_a_low_temperature(lib, rows, dtype):
    """scale 100: log sums of thousands from ordinary logits, rows that are not uniform, both gradients."""
    g = torch.Generator().manual_seed(21)
    x = 15 + (0.05 if dtype == torch.float32 else 0.3) * torch.randn(rows, 9001, generator=g)
    x[1, 40] = 16.5
    x = x.to(dtype)
    tok = torch.randint(0, 9001, (rows,), generator=g)
    tok[1] = 40
    gl, gh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    got, want, logp, h = _gradient_and_formula(x, tok, 100.0, gl, gh)
    p, far = torch.exp(logp), logp.abs()
    e = 2.0 ** -20 + 2.0 ** -22 * (8 + far)
    tol = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22) * want.abs() + 1e-30
    tol = tol + 100 * (gl.double().abs()[:, None] + 4 * gh.double().abs()[:, None] * (1 + far + h)) * e * p
    _near(got, want, tol)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES.keys())
@pytest.mark.parametrize("rows,vocab", [(2, 3001), (2, 40000)])
def test_gradient_where_the_log_sum_leaves_float32(lib, rows, vocab, dtype):
    """scale * logit beyond float32: lse is +-inf, but the row is uniform like any other of equal logits."""
    x = torch.full((rows, vocab), torch.finfo(dtype).min).to(dtype)
    x[1] = torch.finfo(dtype).max
    tok = torch.tensor([7, vocab - 1])
    r = lt.token_logprobs(x.cuda(), tok.cuda(), scale=1.4)
    assert r.lse.tolist() == [NEG_INF, -NEG_INF]
    gl, gh = torch.tensor([2.0, -3.0]), torch.tensor([1.0, -1.0])
    got, want, logp, h = _gradient_and_formula(x, tok, 1.4, gl, gh)
    p = torch.exp(logp)
    e = 2.0 ** -20 + 2.0 ** -22 * (8 + logp.abs())
    tol = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22) * want.abs() + 1e-30
    tol = tol + 1.4 * (gl.double().abs()[:, None] + 4 * gh.double().abs()[:, None] * (1 + logp.abs() + h)) * e * p
    _near(got, want, tol)
    x[0] = NEG_INF                                    # and a row of nothing still has none
    r = lt.token_logprobs(x.cuda(), tok.cuda(), scale=1.4)
    got = lt.token_logprobs_backward(x.cuda(), tok.cuda(), r.lse, r.entropy, gl.cuda(), gh.cuda(), scale=1.4)
    assert (got[0] == 0).all() and torch.isfinite(got[1]).all()
