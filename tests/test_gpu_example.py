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
