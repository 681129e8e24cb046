"""Refusals and workspace sizes of the serving entry points: host checks only,
nothing is enqueued."""
import pytest

from paper_2607_11976_amd import litetopk as lt

P = 256  # an aligned address that is never used


def plan(**over):
    a = dict(ctx=P, new=P, n=4, page=16, table=P, ld=8, width=8, free=P, nfree=9, used=P, cap=32, cu=P, seq=P,
             slots=P, pos=P, out=2 * P, status=P, stream=None)
    a.update(over)
    return lt.lt_paged_plan(*a.values())


@pytest.mark.parametrize("over,code", [
    (dict(n=-1), lt.LT_EINVAL), (dict(page=0), lt.LT_EINVAL), (dict(page=12), lt.LT_EINVAL),
    (dict(page=8192), lt.LT_EINVAL), (dict(ld=7), lt.LT_EINVAL), (dict(nfree=-1), lt.LT_EINVAL),
    (dict(cap=-1), lt.LT_EINVAL), (dict(n=lt.LT_PLAN_MAX_REQUESTS + 1), lt.LT_EUNSUPPORTED),
    (dict(ctx=None), lt.LT_EINVAL), (dict(used=None), lt.LT_EINVAL), (dict(out=P), lt.LT_EINVAL),
    (dict(cu=None), lt.LT_EINVAL), (dict(table=None), lt.LT_EINVAL), (dict(free=None), lt.LT_EINVAL),
    (dict(slots=None), lt.LT_EINVAL), (dict(slots=P + 4), lt.LT_EINVAL)])
def test_plan_refusals(over, code):
    assert plan(**over) == code


def append(**over):
    a = dict(k=P, v=P, dtype=lt.LT_BF16, ks=256, vs=256, rows=3, codes=P, scales=P, pages=4, page=16, heads=2, d=128,
             slots=P, stream=None)
    a.update(over)
    return lt.lt_cache4_append(*a.values())


@pytest.mark.parametrize("over,code", [
    (dict(d=96), lt.LT_EUNSUPPORTED), (dict(d=0), lt.LT_EINVAL), (dict(dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED),
    (dict(rows=-1), lt.LT_EINVAL), (dict(ks=255), lt.LT_EINVAL), (dict(vs=260), lt.LT_EINVAL),
    (dict(k=P + 2), lt.LT_EINVAL), (dict(slots=None), lt.LT_EINVAL), (dict(codes=P + 8), lt.LT_EINVAL),
    (dict(page=3), lt.LT_EINVAL), (dict(heads=0), lt.LT_EINVAL),
    (dict(heads=lt.LT_CACHE4_MAX_HEADS + 1), lt.LT_EUNSUPPORTED), (dict(rows=0), lt.LT_OK)])
def test_append_refusals(over, code):
    assert append(**over) == code


@pytest.mark.parametrize("over,code", [
    (dict(d=96), lt.LT_EUNSUPPORTED), (dict(rows=-1), lt.LT_EINVAL), (dict(slots=None), lt.LT_EINVAL),
    (dict(k=P + 8), lt.LT_EINVAL), (dict(page=24), lt.LT_EINVAL), (dict(rows=0), lt.LT_OK)])
def test_read_refusals(over, code):
    a = dict(codes=P, scales=P, pages=4, page=16, heads=2, d=128, slots=P, rows=3, k=P, v=P, stream=None)
    a.update(over)
    assert lt.lt_cache4_read(*a.values()) == code


def attention(**over):
    a = dict(q=P, qs=2048, tokens=5, hq=16, d=128, codes=P, scales=P, pages=9, page=16, hkv=4, table=P, ld=8, width=8,
             cu=P, seq=P, n=2, start=None, end=None, sel=None, sel_ld=0, k=0, base=None, scale=0.1, out=P, lse=P,
             ws=P, bytes=1 << 40, stream=None)
    a.update(over)
    return lt.lt_cache4_attention(*a.values())


@pytest.mark.parametrize("over,code", [
    (dict(tokens=-1), lt.LT_EINVAL), (dict(hq=15), lt.LT_EINVAL), (dict(d=256), lt.LT_EUNSUPPORTED),
    (dict(q=None), lt.LT_EINVAL), (dict(q=P + 8), lt.LT_EINVAL), (dict(qs=2047), lt.LT_EINVAL),
    (dict(qs=2052), lt.LT_EINVAL), (dict(out=P + 2), lt.LT_EINVAL), (dict(cu=None), lt.LT_EINVAL),
    (dict(seq=None), lt.LT_EINVAL), (dict(table=None), lt.LT_EINVAL), (dict(ld=7), lt.LT_EINVAL),
    (dict(scale=0.0), lt.LT_EINVAL), (dict(scale=-1.0), lt.LT_EINVAL), (dict(scale=float("nan")), lt.LT_EINVAL),
    (dict(scale=float("inf")), lt.LT_EINVAL), (dict(k=4, sel=None, sel_ld=4), lt.LT_EINVAL),
    (dict(k=4, sel=P, sel_ld=3), lt.LT_EINVAL), (dict(k=0, sel=P), lt.LT_EINVAL), (dict(k=-1), lt.LT_EINVAL),
    (dict(ws=None), lt.LT_EINVAL), (dict(ws=P + 16), lt.LT_EINVAL), (dict(bytes=16), lt.LT_EWORKSPACE),
    (dict(pages=0), lt.LT_EINVAL), (dict(page=48), lt.LT_EINVAL),
    (dict(hq=2048, qs=1 << 18), lt.LT_EUNSUPPORTED), (dict(tokens=1 << 27, hq=16), lt.LT_EUNSUPPORTED),
    (dict(tokens=0, q=None, out=None, cu=None), lt.LT_OK)])
def test_attention_refusals(over, code):
    assert attention(**over) == code


def test_attention_workspace_sizes():
    size = lt.lt_cache4_attention_workspace_size
    assert size(1, 1, 8, 1, 128) >= 256 and size(0, 0, 8, 8, 64) > 0
    assert size(1, 1, 8, 3, 128) == 0 and size(1, 1, 8, 8, 80) == 0 and size(-1, 1, 8, 8, 64) == 0
    assert size(32, 32, 64, 1, 128, 2048) > 0 and size(32, 32, 64, 1, 128, -1) == 0


@pytest.mark.parametrize("hq,hkv,d", [(64, 8, 128), (8, 8, 64), (64, 1, 128), (12, 4, 64)])
def test_attention_workspace_serves_smaller_calls(hq, hkv, d):
    size = lt.lt_cache4_attention_workspace_size
    counts = [0, 1, 2, 3, 8, 15, 16, 17, 64, 65, 128, 129, 255, 256, 257, 2048, 70000]
    for k in (0, 1, 130, 2048):
        for r in range(len(counts) - 1):
            for t in range(len(counts) - 1):
                at = size(counts[t], counts[r], hq, hkv, d, k)
                assert at > 0
                assert at <= size(counts[t + 1], counts[r], hq, hkv, d, k)
                assert at <= size(counts[t], counts[r + 1], hq, hkv, d, k)
        assert k == 0 or size(256, 7, hq, hkv, d, k) <= size(256, 7, hq, hkv, d, 2 * k)


def logprobs(**over):
    a = dict(x=P, dtype=lt.LT_BF16, ld=100, rows=3, vocab=100, tok=P, scale=1.0, top=5, lp=P, h=P, lse=P, ti=P, tl=P,
             ws=P, bytes=1 << 40, stream=None)
    a.update(over)
    return lt.lt_token_logprobs(*a.values())


@pytest.mark.parametrize("over,code", [
    (dict(dtype=lt.LT_FP8_E4M3FN), lt.LT_EUNSUPPORTED), (dict(ld=99), lt.LT_EINVAL), (dict(rows=-1), lt.LT_EINVAL),
    (dict(scale=0.0), lt.LT_EINVAL), (dict(scale=float("nan")), lt.LT_EINVAL), (dict(top=-1), lt.LT_EINVAL),
    (dict(top=lt.LT_LOGPROB_MAX_TOP + 1), lt.LT_EUNSUPPORTED), (dict(ti=None), lt.LT_EINVAL),
    (dict(x=None), lt.LT_EINVAL), (dict(x=P + 1), lt.LT_EINVAL), (dict(tok=None), lt.LT_EINVAL),
    (dict(lse=None), lt.LT_EINVAL), (dict(bytes=0), lt.LT_EWORKSPACE), (dict(ws=P + 8), lt.LT_EINVAL),
    (dict(vocab=lt.LT_LOGPROB_MAX_VOCAB + 1, ld=1 << 31), lt.LT_EUNSUPPORTED), (dict(rows=0), lt.LT_OK)])
def test_logprob_refusals(over, code):
    assert logprobs(**over) == code


@pytest.mark.parametrize("over,code", [
    (dict(ld=99), lt.LT_EINVAL), (dict(out_ld=99), lt.LT_EINVAL), (dict(scale=-1.0), lt.LT_EINVAL),
    (dict(lse=None), lt.LT_EINVAL), (dict(out=None), lt.LT_EINVAL), (dict(dtype=7), lt.LT_EUNSUPPORTED),
    (dict(rows=0), lt.LT_OK)])
def test_logprob_backward_refusals(over, code):
    a = dict(x=P, dtype=lt.LT_F32, ld=100, rows=3, vocab=100, tok=P, scale=1.0, lse=P, h=P, gl=P, gh=None, out=P,
             out_ld=100, stream=None)
    a.update(over)
    assert lt.lt_token_logprobs_backward(*a.values()) == code


def test_logprob_workspace_sizes():
    size = lt.lt_token_logprobs_workspace_size
    assert size(lt.LT_F32, 1, 100000, 20) > size(lt.LT_F32, 4096, 1000, 20) >= 256
    assert size(lt.LT_FP8_E4M3FN, 1, 10, 1) == 0 and size(lt.LT_F32, 1, 10, lt.LT_LOGPROB_MAX_TOP + 1) == 0


@pytest.mark.parametrize("dtype", [lt.LT_F32, lt.LT_BF16])
def test_logprob_workspace_serves_smaller_calls(dtype):
    """Sizes rise with rows, entries and alternatives."""
    size = lt.lt_token_logprobs_workspace_size
    rows = [0, 1, 2, 3, 7, 8, 31, 32, 33, 64, 100, 500, 1000, 1023, 1024, 1025, 2039, 5000, 100000]
    vocabs = [0, 1, 1000, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 32000, 50257, 128001, 131072, 262144, 10**7,
              2**30]
    for top in (0, 1, 64):
        for i in range(len(rows) - 1):
            for j in range(len(vocabs) - 1):
                at = size(dtype, rows[i], vocabs[j], top)
                assert at >= 256
                assert at <= size(dtype, rows[i + 1], vocabs[j], top)
                assert at <= size(dtype, rows[i], vocabs[j + 1], top)
                assert at <= size(dtype, rows[i], vocabs[j], 64)


def test_attention_lists_of_too_many_entries():
    """Places in a list are 32-bit, and a step may look some way past its end."""
    most = 0x7FFF0000
    for k in (most + 1, 2**31 - 64, 2**31 - 1):
        assert attention(k=k, sel=P, sel_ld=2**31) == lt.LT_EUNSUPPORTED
        assert lt.lt_cache4_attention_workspace_size(5, 2, 16, 4, 128, k) == 0
    assert lt.lt_cache4_attention_workspace_size(5, 2, 16, 4, 128, most) > 0
    assert attention(k=most, sel=P, sel_ld=2**31, bytes=16) == lt.LT_EWORKSPACE


def test_calls_of_more_threads_than_a_launch_counts():
    """2^32 threads of a launch: refused on the host, the largest sizes below pass these checks."""
    for n, code in ((2**25, lt.LT_EUNSUPPORTED), (2**25 - 2, lt.LT_EINVAL)):   # x 8 heads x 16 chunks of 8 values
        assert append(rows=n, heads=8, ks=1024, vs=1024, slots=None) == code
        assert lt.lt_cache4_read(P, P, 4, 16, 8, 128, None, n, P, P, None) == code
    size = lt.lt_cache4_attention_workspace_size
    assert size(2**24 - 1, 2, 1, 1, 64, 100) > 0 and size(2**24, 2, 1, 1, 64, 100) == 0    # a block a token
    assert size(2**24, 2, 1, 1, 64, 0) > 0
    assert attention(tokens=2**24, hq=1, hkv=1, k=4, sel=P, sel_ld=4) == lt.LT_EUNSUPPORTED
    assert logprobs(rows=lt.LT_LOGPROB_MAX_ROWS + 1) == lt.LT_EUNSUPPORTED
    assert logprobs(rows=lt.LT_LOGPROB_MAX_ROWS, bytes=0) == lt.LT_EWORKSPACE
    assert lt.lt_token_logprobs_workspace_size(lt.LT_F32, lt.LT_LOGPROB_MAX_ROWS + 1, 100, 5) == 0
    assert lt.lt_token_logprobs_backward(P, lt.LT_F32, 100, lt.LT_LOGPROB_MAX_ROWS + 1, 100, P, 1.0, P, P, P, None, P,
                                         100, None) == lt.LT_EUNSUPPORTED


@pytest.mark.parametrize("scale,code", [(3.0e38, lt.LT_EINVAL), (2.4e38, lt.LT_EINVAL), (2.3e38, lt.LT_EWORKSPACE),
                                        (1e-45, lt.LT_EWORKSPACE)])
def test_scales_times_log2_e_are_finite(scale, code):
    """Scores are taken in powers of two: a scale that overflows there made every result NaN."""
    assert attention(scale=scale, bytes=16) == code
    assert logprobs(scale=scale, bytes=0) == code
    none = lt.lt_token_logprobs_backward(P, lt.LT_F32, 100, 0, 100, P, scale, P, P, P, None, P, 100, None)
    assert none == (lt.LT_OK if code == lt.LT_EWORKSPACE else lt.LT_EINVAL)


@pytest.mark.parametrize("over", [dict(seq="ctx"), dict(status="new"), dict(cu="new"), dict(out="used"), dict(seq="used"),
                                  dict(pos="free"), dict(slots="free"), dict(status="ctx")])
def test_plan_results_in_place_of_inputs(over):
    """Blocks read the lengths while others write results: a result there would be read as a length."""
    names = ("ctx", "new", "table", "free", "used", "cu", "seq", "slots", "pos", "out", "status")
    own = {n: (i + 1) << 20 for i, n in enumerate(names)}
    own.update({n: own[o] for n, o in over.items()})
    assert plan(**own) == lt.LT_EINVAL
