"""Refusals and workspace sizes of rotary positions, rotated cache writes, beam
selection and reordered pages (host checks only, nothing is enqueued), and the
frequencies of scaled contexts."""
import math

import pytest
import torch

from paper_2607_11976_amd import litetopk as lt

P = 256  # an aligned address that is never used
INF = float("inf")
NAN = float("nan")


def rotary(**over):
    a = dict(x=P, dtype=lt.LT_BF16, ts=1024, hs=128, tokens=3, heads=8, d=128, pos=P, freq=P, pairs=64, start=0, amp=1.0,
             flags=0, out=2 * P, out_dtype=lt.LT_BF16, ots=1024, ohs=128, stream=None)
    a.update(over)
    return lt.lt_rotary(*a.values())


@pytest.mark.parametrize("over,code", [
    (dict(dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED), (dict(out_dtype=lt.LT_F32), lt.LT_EUNSUPPORTED),
    (dict(out_dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED), (dict(d=1025, ts=9000, hs=1025), lt.LT_EUNSUPPORTED),
    (dict(tokens=-1), lt.LT_EINVAL), (dict(heads=-1), lt.LT_EINVAL), (dict(d=0), lt.LT_EINVAL),
    (dict(pairs=65), lt.LT_EINVAL), (dict(pairs=-1), lt.LT_EINVAL), (dict(start=-1), lt.LT_EINVAL),
    (dict(start=1), lt.LT_EINVAL), (dict(pairs=0x7FFFFFFF), lt.LT_EINVAL), (dict(amp=INF), lt.LT_EINVAL),
    (dict(amp=NAN), lt.LT_EINVAL), (dict(flags=4), lt.LT_EINVAL), (dict(x=None), lt.LT_EINVAL),
    (dict(x=P + 1), lt.LT_EINVAL), (dict(pos=None), lt.LT_EINVAL), (dict(pos=P + 2), lt.LT_EINVAL),
    (dict(freq=None), lt.LT_EINVAL), (dict(freq=P + 1), lt.LT_EINVAL), (dict(out=None), lt.LT_EINVAL),
    (dict(out=2 * P + 1), lt.LT_EINVAL), (dict(ts=-1), lt.LT_EINVAL), (dict(ohs=127), lt.LT_EINVAL),
    (dict(ots=127), lt.LT_EINVAL), (dict(ots=1023), lt.LT_EINVAL), (dict(ots=128, ohs=128), lt.LT_EINVAL),
    (dict(out=P, ts=2048), lt.LT_EINVAL), (dict(out=P, hs=256, ts=2048, ots=2048), lt.LT_EINVAL),
    (dict(out=P, dtype=lt.LT_F32), lt.LT_EINVAL), (dict(tokens=0), lt.LT_OK), (dict(heads=0), lt.LT_OK),
    (dict(tokens=0x7FFFFFFF, heads=1024, ts=1 << 20, ots=1 << 20), lt.LT_EUNSUPPORTED),
    (dict(heads=lt.LT_ROTARY_MAX_HEADS + 1, ts=1 << 28, ots=1 << 28), lt.LT_EUNSUPPORTED),
    (dict(ts=(1 << 31) + 1), lt.LT_EINVAL), (dict(hs=1 << 40), lt.LT_EINVAL), (dict(ots=1 << 62), lt.LT_EINVAL),
    (dict(ohs=1 << 62, tokens=1 << 30), lt.LT_EINVAL), (dict(out=3 * P, pos=3 * P), lt.LT_EINVAL),
    (dict(out=3 * P, freq=3 * P), lt.LT_EINVAL)])
def test_rotary_refusals(over, code):
    assert rotary(**over) == code


@pytest.mark.parametrize("over,code", [
    (dict(dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED), (dict(flags=4), lt.LT_EINVAL), (dict(codes=None), lt.LT_EINVAL),
    (dict(scales=None), lt.LT_EINVAL), (dict(scales=P + 2), lt.LT_EINVAL), (dict(codes=P), lt.LT_EINVAL),
    (dict(start=120), lt.LT_EINVAL), (dict(d=2000, pairs=0), lt.LT_EUNSUPPORTED), (dict(tokens=0), lt.LT_OK),
    (dict(scales=P), lt.LT_EINVAL), (dict(scales=2 * P), lt.LT_EINVAL), (dict(pos=2 * P), lt.LT_EINVAL),
    (dict(freq=3 * P), lt.LT_EINVAL)])
def test_rotary_fp8_refusals(over, code):
    a = dict(x=P, dtype=lt.LT_BF16, ts=1024, hs=128, tokens=3, heads=8, d=128, pos=P, freq=P, pairs=64, start=0, amp=1.0,
             flags=0, codes=2 * P, scales=3 * P, stream=None)
    a.update(over)
    assert lt.lt_rotary_fp8(*a.values()) == code


@pytest.mark.parametrize("over,code", [
    (dict(d=96), lt.LT_EUNSUPPORTED), (dict(dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED), (dict(rows=-1), lt.LT_EINVAL),
    (dict(ks=255), lt.LT_EINVAL), (dict(vs=260), lt.LT_EINVAL), (dict(k=P + 2), lt.LT_EINVAL),
    (dict(slots=None), lt.LT_EINVAL), (dict(codes=P + 8), lt.LT_EINVAL), (dict(page=3), lt.LT_EINVAL),
    (dict(pos=None), lt.LT_EINVAL), (dict(pos=P + 2), lt.LT_EINVAL), (dict(freq=None), lt.LT_EINVAL),
    (dict(pairs=65), lt.LT_EINVAL), (dict(start=2), lt.LT_EINVAL), (dict(flags=2), lt.LT_EINVAL),
    (dict(amp=NAN), lt.LT_EINVAL), (dict(q=None), lt.LT_EINVAL), (dict(hq=0), lt.LT_EINVAL),
    (dict(hq=-1), lt.LT_EINVAL), (dict(hq=lt.LT_CACHE4_MAX_HEADS + 1), lt.LT_EUNSUPPORTED),
    (dict(q_out=None), lt.LT_EINVAL), (dict(q_out=P + 8), lt.LT_EINVAL), (dict(q_out=4 * P), lt.LT_EINVAL),
    (dict(qs=1023), lt.LT_EINVAL), (dict(q=P + 1), lt.LT_EINVAL), (dict(rows=0), lt.LT_OK),
    (dict(pages=0, q=None, hq=0), lt.LT_OK), (dict(rows=0x7FFFFFFF, qs=8192, hq=64), lt.LT_EUNSUPPORTED)])
def test_append_rotary_refusals(over, code):
    a = dict(k=P, v=P, dtype=lt.LT_BF16, ks=256, vs=256, rows=3, codes=P, scales=P, pages=4, page=16, heads=2, d=128,
             slots=P, pos=P, freq=P, pairs=64, start=0, amp=1.0, flags=0, q=4 * P, qs=1024, hq=8, q_out=8 * P,
             stream=None)
    a.update(over)
    assert lt.lt_cache4_append_rotary(*a.values()) == code


@pytest.mark.parametrize("name", ["k", "v", "slots", "pos", "freq", "codes", "scales", "q"])
def test_append_rotary_refuses_queries_in_the_place_of_another_argument(name):
    """Blocks of one launch write the queries while others read the rest, or write the cache."""
    a = dict(k=P, v=2 * P, dtype=lt.LT_BF16, ks=256, vs=256, rows=3, codes=3 * P, scales=4 * P, pages=4, page=16, heads=2,
             d=128, slots=5 * P, pos=6 * P, freq=7 * P, pairs=64, start=0, amp=1.0, flags=0, q=8 * P, qs=1024, hq=8,
             q_out=9 * P, stream=None)
    a["q_out"] = a[name]
    assert lt.lt_cache4_append_rotary(*a.values()) == lt.LT_EINVAL


@pytest.mark.parametrize("over,code", [
    (dict(dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED), (dict(batch=-1), lt.LT_EINVAL), (dict(beams=0), lt.LT_EINVAL),
    (dict(top=0), lt.LT_EINVAL), (dict(top=65), lt.LT_EUNSUPPORTED), (dict(vocab=-1), lt.LT_EINVAL),
    (dict(beams=1025), lt.LT_EUNSUPPORTED), (dict(vocab=lt.LT_LOGPROB_MAX_VOCAB + 1, ld=1 << 40), lt.LT_EUNSUPPORTED),
    (dict(batch=1 << 20, beams=64), lt.LT_EUNSUPPORTED), (dict(ld=999), lt.LT_EINVAL), (dict(scale=0.0), lt.LT_EINVAL),
    (dict(scale=-1.0), lt.LT_EINVAL), (dict(scale=NAN), lt.LT_EINVAL), (dict(scale=INF), lt.LT_EINVAL),
    (dict(scale=3e38), lt.LT_EINVAL), (dict(scale=1e300), lt.LT_EINVAL), (dict(scale=7e-31), lt.LT_EINVAL),
    (dict(logits=None), lt.LT_EINVAL),
    (dict(logits=P + 1), lt.LT_EINVAL), (dict(cum=None), lt.LT_EINVAL), (dict(score=None), lt.LT_EINVAL),
    (dict(beam=None), lt.LT_EINVAL), (dict(token=None), lt.LT_EINVAL), (dict(score=P), lt.LT_EINVAL),
    (dict(ws=None), lt.LT_EINVAL), (dict(ws=P + 8), lt.LT_EINVAL), (dict(bytes=16), lt.LT_EWORKSPACE),
    (dict(batch=0), lt.LT_OK)])
def test_beam_refusals(over, code):
    a = dict(logits=P, dtype=lt.LT_BF16, ld=1000, batch=3, beams=4, vocab=1000, cum=P, scale=1.0, top=8, score=2 * P,
             beam=3 * P, token=4 * P, ws=P, bytes=1 << 40, stream=None)
    a.update(over)
    assert lt.lt_beam_select(*a.values()) == code


@pytest.mark.parametrize("one,other", [
    ("score", "beam"), ("score", "token"), ("beam", "token"), ("score", "logits"), ("beam", "logits"), ("token", "logits"),
    ("score", "cum"), ("beam", "cum"), ("token", "cum"), ("score", "ws"), ("beam", "ws"), ("token", "ws"),
    ("ws", "logits"), ("ws", "cum")])
def test_beam_refuses_results_in_the_place_of_another_argument(one, other):
    """A request's block writes its results while others read theirs."""
    a = dict(logits=P, dtype=lt.LT_BF16, ld=1000, batch=3, beams=4, vocab=1000, cum=2 * P, scale=1.0, top=8, score=3 * P,
             beam=4 * P, token=5 * P, ws=6 * P, bytes=1 << 40, stream=None)
    a[one] = a[other]
    assert lt.lt_beam_select(*a.values()) == lt.LT_EINVAL


def test_beam_workspace_sizes():
    size = lt.lt_beam_select_workspace_size
    assert size(lt.LT_BF16, 3, 4, 1000, 65) == 0 and size(lt.LT_FP8_E4M3FN, 3, 4, 1000, 8) == 0
    assert size(lt.LT_BF16, 0, 4, 1000, 8) > 0
    for dtype in (lt.LT_F32, lt.LT_BF16):
        for big in [(1, 1, 260000, 64), (64, 8, 131072, 16), (7, 5, 1000, 3), (3000, 16, 32000, 32)]:
            most = size(dtype, *big)
            for batch in {1, 2, big[0] // 2, big[0]} - {0}:
                for beams in {1, big[1] // 2, big[1]} - {0}:
                    for vocab in {0, 1, 777, big[2] // 2, big[2]}:
                        if vocab <= big[2] and batch <= big[0]:
                            assert 0 < size(dtype, batch, beams, vocab, big[3]) <= most


@pytest.mark.parametrize("over,code", [
    (dict(rows=-4), lt.LT_EINVAL), (dict(rows=7), lt.LT_EINVAL), (dict(group=0), lt.LT_EINVAL),
    (dict(group=65, rows=65), lt.LT_EUNSUPPORTED), (dict(rows=lt.LT_PLAN_MAX_REQUESTS + 4), lt.LT_EUNSUPPORTED),
    (dict(width=-1), lt.LT_EINVAL), (dict(ld=8), lt.LT_EINVAL), (dict(new_ld=8), lt.LT_EINVAL),
    (dict(page=12), lt.LT_EINVAL), (dict(nfree=-1), lt.LT_EINVAL), (dict(lens=None), lt.LT_EINVAL),
    (dict(parents=None), lt.LT_EINVAL), (dict(table=None), lt.LT_EINVAL), (dict(new_table=None), lt.LT_EINVAL),
    (dict(free=None), lt.LT_EINVAL), (dict(used=None), lt.LT_EINVAL), (dict(used_out=None), lt.LT_EINVAL),
    (dict(status=None), lt.LT_EINVAL), (dict(copies=None), lt.LT_EINVAL), (dict(new_lens=None), lt.LT_EINVAL),
    (dict(new_table=P), lt.LT_EINVAL), (dict(new_lens=2 * P), lt.LT_EINVAL), (dict(used_out=5 * P), lt.LT_EINVAL),
    (dict(status=3 * P), lt.LT_EINVAL), (dict(copies=6 * P), lt.LT_EINVAL), (dict(free=6 * P), lt.LT_EINVAL),
    (dict(free=P), lt.LT_EINVAL), (dict(free=2 * P), lt.LT_EINVAL), (dict(keep=5 * P), lt.LT_EINVAL),
    (dict(ws=None), lt.LT_EINVAL), (dict(ws=P + 8), lt.LT_EINVAL), (dict(bytes=16), lt.LT_EWORKSPACE),
    (dict(width=1 << 28, ld=1 << 28, new_ld=1 << 28), lt.LT_EUNSUPPORTED)])
def test_reorder_refusals(over, code):
    a = dict(table=P, ld=9, width=9, lens=2 * P, parents=3 * P, rows=8, group=4, page=16, keep=4 * P, free=5 * P,
             nfree=50, used=6 * P, new_table=7 * P, new_ld=9, new_lens=8 * P, copies=9 * P, used_out=10 * P,
             status=11 * P, ws=12 * P, bytes=1 << 40, stream=None)
    a.update(over)
    assert lt.lt_paged_reorder(*a.values()) == code


RESULTS = ["new_table", "new_lens", "copies", "used_out", "status"]
READ = ["table", "lens", "parents", "keep", "used", "free"]


@pytest.mark.parametrize("one,other", [(o, r) for i, o in enumerate(RESULTS) for r in RESULTS[i + 1:]]
                         + [("ws", n) for n in RESULTS + READ])
def test_reorder_refuses_results_in_the_place_of_another_argument(one, other):
    a = dict(table=P, ld=9, width=9, lens=2 * P, parents=3 * P, rows=8, group=4, page=16, keep=4 * P, free=5 * P,
             nfree=50, used=6 * P, new_table=7 * P, new_ld=9, new_lens=8 * P, copies=9 * P, used_out=10 * P,
             status=11 * P, ws=12 * P, bytes=1 << 40, stream=None)
    a[one] = a[other]
    assert lt.lt_paged_reorder(*a.values()) == lt.LT_EINVAL


def test_reorder_workspace_sizes():
    size = lt.lt_paged_reorder_workspace_size
    assert size(-1) == 0 and size(lt.LT_PLAN_MAX_REQUESTS + 1) == 0
    sizes = [size(n) for n in range(0, lt.LT_PLAN_MAX_REQUESTS + 1, 61)]
    assert sizes[0] > 0 and sizes == sorted(sizes)


@pytest.mark.parametrize("over,code", [
    (dict(n=-1), lt.LT_EINVAL), (dict(copies=None), lt.LT_EINVAL), (dict(d=32), lt.LT_EUNSUPPORTED),
    (dict(page=24), lt.LT_EINVAL), (dict(codes=P + 4), lt.LT_EINVAL), (dict(n=0), lt.LT_OK), (dict(pages=0), lt.LT_OK),
    (dict(n=0x7FFFFFFF, heads=1024, page=4096), lt.LT_EUNSUPPORTED)])
def test_copy_refusals(over, code):
    a = dict(codes=P, scales=P, pages=4, page=16, heads=2, d=128, copies=P, n=5, stream=None)
    a.update(over)
    assert lt.lt_cache4_copy(*a.values()) == code


# ---- frequencies -----------------------------------------------------------

def _f(**kw):
    return lt.rotary_frequencies(device="cpu", **kw)


def test_frequencies():
    r = _f(dim=8, base=100.0)
    want = [1.0, 100.0 ** -0.25, 0.1, 100.0 ** -0.75]
    assert r.inv_freq.dtype == torch.float32 and r.amplitude == 1.0 and r.start == 0 and not r.interleaved
    assert torch.equal(r.inv_freq, torch.tensor(want, dtype=torch.float64).float())
    assert torch.equal(_f(dim=8, base=100.0, method="linear", factor=4.0).inv_freq,
                       (torch.tensor(want, dtype=torch.float64) / 4).float())
    ntk = _f(dim=8, base=100.0, method="base", factor=4.0).inv_freq
    assert ntk[0] == 1.0 and abs(float(ntk[3]) * 4 / want[3] - 1) < 1e-6


@pytest.mark.parametrize("method,amplitude", [("ramp", 0.1 * math.log(8.0) + 1.0), ("turns", 1.0)])
def test_frequencies_between(method, amplitude):
    dim, n, factor = 128, 4096, 8.0
    plain = _f(dim=dim).inv_freq.double()
    r = _f(dim=dim, method=method, factor=factor, original_length=n)
    share = (r.inv_freq.double() / plain - 1 / factor) / (1 - 1 / factor)   # 1: as it was, 0: divided
    assert abs(r.amplitude - amplitude) < 1e-12
    turns = n * plain / (2 * math.pi)
    high = 32.0 if method == "ramp" else 4.0
    # the ramp's ends are whole indices, one step past the exact ones at most
    step = 10000.0 ** (2 / dim) if method == "ramp" else 1.0
    assert torch.all(share[turns > high * step] > 1 - 1e-6) and torch.all(share[turns < 1 / step] < 1e-6)
    assert torch.all(share[1:] <= share[:-1] + 1e-6) and ((share > 0.01) & (share < 0.99)).any()
    assert _f(dim=dim, method=method, factor=factor, original_length=n, amplitude=2.0).amplitude == 2.0


@pytest.mark.parametrize("kw", [dict(dim=7), dict(dim=0), dict(dim=8, base=0.0), dict(dim=8, method="other"),
                                dict(dim=2, method="base", factor=2.0), dict(dim=8, method="ramp", factor=2.0),
                                dict(dim=8, method="turns", factor=2.0, original_length=9, low=4.0, high=4.0),
                                dict(dim=8, factor=0.0)])
def test_frequencies_that_make_no_sense(kw):
    with pytest.raises(lt.LiteTopKError):
        _f(**kw)
