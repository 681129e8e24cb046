"""The decoding example: sparse decoding with lists longer than the contexts is
dense decoding, and its tokens are the best ones of its logits."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def _prompts():
    g = torch.Generator().manual_seed(3)
    return [torch.randint(0, 4096, (n,), generator=g).tolist() for n in (33, 5, 70)]


def test_lists_of_all_keys_decode_as_dense_attention(lib):
    import decode_step
    a = decode_step.generate(_prompts(), steps=6, selected=128, sparse=True)
    b = decode_step.generate(_prompts(), steps=6, sparse=False)
    assert torch.equal(a[0], b[0])
    # outputs in bfloat16 feed logits of order 1: 2^-8 of them, once more for the layer's sums
    assert torch.allclose(a[1], b[1], atol=2e-2) and torch.allclose(a[2], b[2], atol=2e-2)


def test_short_lists_run_and_repeat(lib):
    import decode_step
    a = decode_step.generate(_prompts(), steps=5, selected=16)
    b = decode_step.generate(_prompts(), steps=5, selected=16)
    assert torch.equal(a[0], b[0])
    assert (a[1] <= 0).all() and (a[2] >= 0).all()


def test_log_probabilities_of_a_step(lib):
    import decode_step
    from paper_2607_11976_amd import litetopk as lt
    w = decode_step.weights()
    dec = decode_step.Decoder(w, 3, 90, 32)
    p = _prompts()
    lens = torch.tensor([len(x) for x in p], dtype=torch.int32, device="cuda")
    logits = dec.step(torch.tensor([t for x in p for t in x], device="cuda"), lens, sparse=False)
    r = lt.token_logprobs(logits, torch.tensor([1, 2, 3], device="cuda"), top=2)
    want = torch.log_softmax(logits.double(), -1)
    assert torch.allclose(r.logprob.double(), want[torch.arange(3), torch.tensor([1, 2, 3])], atol=1e-5)
    assert torch.equal(r.top_index.long(), want.topk(2, -1).indices)


def test_a_step_without_room_is_an_error(lib):
    import decode_step
    dec = decode_step.Decoder(decode_step.weights(), 3, 40, 32)
    before = dec.lens.clone()
    p = _prompts()                                  # the last is longer than 40
    lens = torch.tensor([len(x) for x in p], dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError, match=r"\[2\]"):
        dec.step(torch.tensor([t for x in p for t in x], device="cuda"), lens, sparse=False)
    assert torch.equal(dec.lens, before) and int(dec.used) == 0


def test_tokens_without_slots_see_nothing_by_their_visible_ends(lib):
    """The plan's outputs as visible ends: a request that got no pages gives zeros, the others their attention."""
    from paper_2607_11976_amd import litetopk as lt
    i = dict(dtype=torch.int32, device="cuda")
    codes, scales = lt.cache4_empty(6, 16, 2, 64)
    table = torch.tensor([[0, -1], [1, -1], [2, -1]], **i)
    plan = lt.paged_plan(torch.tensor([10, 15, 3], **i), torch.tensor([2, 4, 5], **i), table, torch.tensor([3], **i),
                         torch.tensor([1], **i), 16, 12)
    assert plan.status.tolist() == [0, 2, 0] and plan.slots[2:6].tolist() == [-1] * 4
    kv = torch.randn(2, 12, 2, 64, device="cuda")
    old = torch.arange(96, device="cuda")
    lt.cache4_append(torch.randn(96, 2, 64, device="cuda"), torch.randn(96, 2, 64, device="cuda"), codes, scales, old)
    lt.cache4_append(kv[0], kv[1], codes, scales, plan.slots)
    q = torch.randn(12, 4, 64, device="cuda").to(torch.bfloat16)
    end = torch.where(plan.slots >= 0, plan.positions + 1, torch.zeros_like(plan.positions))
    out, lse = lt.cache4_attention(q, codes, scales, table, plan.cu_tokens, plan.seq_lens, visible_end=end)
    assert (out[2:6] == 0).all() and (lse[2:6] == float("-inf")).all()
    want = lt.cache4_attention(q, codes, scales, table, plan.cu_tokens, plan.seq_lens)
    for part in (slice(0, 2), slice(6, 11)):
        assert torch.equal(out[part], want[0][part]) and torch.equal(lse[part], want[1][part])
    assert torch.isfinite(want[0][2:6]).all() and (want[0][2:6] != 0).any()     # what the default would have given
