"""GPU: arrays whose offsets pass 32 bits. What lies at their far end is compared with
the same rows in a call of their own (which the other tests compare with the
definitions)."""
import pytest
import torch

from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu


def _rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def test_rotary_past_32_bits(lib):
    tokens, heads, d = 36000, 512, 128                  # 2.36e9 values
    x = torch.zeros(tokens, heads, d, dtype=torch.bfloat16, device="cuda")
    x[-3:] = _rand(1, 3, heads, d).to(torch.bfloat16)
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    rot = lt.rotary_frequencies(d)
    small = lt.rotary(x[-3:], pos[-3:], rot)
    codes, scales = lt.rotary_fp8(x[-3:], pos[-3:], rot)
    far_codes, far_scales = lt.rotary_fp8(x, pos, rot)
    assert torch.equal(far_codes[-3:].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(far_scales[-3:], scales)
    assert not (far_codes[:-3].view(torch.uint8) & 0x7F).any()     # zeros of either sign
    lt.rotary(x, pos, rot, out=x)
    assert torch.equal(x[-3:], small) and not x[:-3].any()


def test_cache_past_32_bits(lib):
    pages, page, heads, d = 70000, 64, 8, 128           # 4.6e9 bytes of codes
    codes, scales = lt.cache4_empty(pages, page, heads, d)
    k, v = _rand(2, 5, heads, d), _rand(3, 5, heads, d)
    pos = torch.arange(5, dtype=torch.int32, device="cuda") + 1000
    slots = torch.tensor([0, 1, pages * page - 1, pages * page // 2, (pages - 1) * page], device="cuda")
    rot = lt.rotary_frequencies(d)
    lt.cache4_append_rotary(k, v, codes, scales, slots, pos, rot)
    small = lt.cache4_empty(1, page, heads, d)
    lt.cache4_append_rotary(k, v, *small, torch.arange(5, device="cuda"), pos, rot)
    for a, b in zip(lt.cache4_read(codes, scales, slots), lt.cache4_read(*small, torch.arange(5, device="cuda"))):
        assert torch.equal(a, b)
    lt.cache4_copy(codes, scales, torch.tensor([[pages - 1, 7], [0, pages - 2]], dtype=torch.int32, device="cuda"))
    assert torch.equal(codes[7], codes[pages - 1]) and torch.equal(scales[7], scales[pages - 1])
    assert torch.equal(codes[pages - 2], codes[0]) and torch.equal(scales[pages - 2], scales[0])
    assert codes[7].any() and codes[0].any() and not codes[8].any()


def test_logits_past_32_bits(lib):
    reqs, beams, vocab = 4500, 4, 131072                # 2.36e9 logits
    x = torch.zeros(reqs * beams, vocab, dtype=torch.bfloat16, device="cuda")
    x[-beams:] = _rand(4, beams, vocab).to(torch.bfloat16)
    cum = torch.full((reqs, beams), float("-inf"), device="cuda")
    cum[0], cum[-1] = -1.0, _rand(5, beams)
    r = lt.beam_select(x, cum, 8)
    small = lt.beam_select(x[-beams:], cum[-1:], 8)
    assert all(torch.equal(a[-1:], b) for a, b in zip(r, small))
    assert torch.all(r.beam[1:-1] == -1) and r.token[0].tolist() == list(range(8)) and not r.beam[0].any()
