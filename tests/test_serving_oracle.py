"""CPU pins of the serving oracle: hand-worked plans and codes, the attention
definition against a direct sum, and the log probabilities' gradient against
central differences."""
import math

import pytest
import torch

from oracle import serving_oracle as orc


def test_plan_by_hand():
    # pages of 4; request 0 fills its page and takes one more, 1 is idle, 2 starts
    # empty and needs two, 3 needs more pages than its row has, 4 needs none
    p = orc.paged_plan([3, 5, 0, 6, 1], [2, 0, 7, 9, 2], [[8, -1, -1], [2, 3, -1], [-1, -1, -1], [4, 5, -1],
                                                         [7, -1, -1]], [9, 1, 0, 6], 1, 4, 24)
    assert p["status"] == [0, 0, 0, 1, 0]
    assert p["free_used"] == [4]
    assert p["table"] == [[8, 1, -1], [2, 3, -1], [0, 6, -1], [4, 5, -1], [7, -1, -1]]
    assert p["cu_tokens"] == [0, 2, 2, 9, 18, 20] and p["seq_lens"] == [5, 5, 7, 6, 3]
    assert p["slots"][:9] == [35, 4, 0, 1, 2, 3, 24, 25, 26]
    assert p["slots"][9:18] == [-1] * 9 and p["slots"][18:] == [29, 30] + [-1] * 4
    assert p["positions"] == [3, 4, 0, 1, 2, 3, 4, 5, 6] + list(range(6, 15)) + [1, 2] + [-1] * 4


def test_plan_out_of_pages_stays_closed():
    p = orc.paged_plan([0, 0, 1, 0], [4, 9, 1, 4], [[-1] * 3, [-1] * 3, [5, -1, -1], [-1] * 3], [1, 2, 3], 0, 4, 20)
    assert p["status"] == [0, 2, 0, 2] and p["free_used"] == [1]


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.0000001, 1), (6.0, 0), (3.5, -1), (3.6, 0), (0.0, -127),
                                   (1e-45, -127), (2.9e38, 125), (3.4028235e38, 125)])
def test_block_exponent(top, e):
    assert orc.block_exponent(top) == e
    assert (top <= 7 * math.ldexp(1.0, e) or e == 125) and (e == -127 or top > 7 * math.ldexp(1.0, e - 1))


def test_codes_by_hand():
    x = torch.zeros(1, 32)
    x[0, :12] = torch.tensor([7.0, 5.0, -2.5, 0.25, 0.75, -0.2, 3.5, 1.25, 1.75, -6.5, 0.26, 0.0])
    codes, scales = orc.quantise(x)
    assert scales.tolist() == [[127]]
    got = orc.decode(codes, scales)[0, :12]
    assert got.tolist() == [6.0, 4.0, -2.0, 0.0, 1.0, -0.0, 4.0, 1.0, 2.0, -6.0, 0.5, 0.0]
    assert codes[0, 0].item() == 7 | (6 << 4)  # the earlier value is the low half
    x[0, 3] = float("inf")
    codes, scales = orc.quantise(x)
    assert scales.tolist() == [[255]] and torch.isnan(orc.decode(codes, scales)).all()


def test_attention_by_direct_sum():
    g = torch.Generator().manual_seed(1)
    codes = torch.randint(0, 256, (3, 1, 4, 2, 32), generator=g, dtype=torch.uint8)
    scales = torch.randint(124, 128, (3, 1, 4, 2, 2), generator=g, dtype=torch.uint8)
    q = torch.randn(2, 2, 64, generator=g)
    table = torch.tensor([[2, 0]])
    out, lse, _ = orc.attention(q, codes, scales, table, [0, 2], [6], 0.3)
    kv = orc.decode(codes, scales)
    for t in range(2):
        for h in range(2):
            num, den = torch.zeros(64, dtype=torch.float64), 0.0
            for j in range(5 + t):                       # causal: 6 keys, the last two are the new tokens
                k, v = kv[table[0, j // 4], 0, j % 4]
                w = math.exp(0.3 * float(k @ q[t, h].double()))
                num, den = num + w * v, den + w
            assert torch.allclose(out[t, h], num / den, rtol=1e-12)
            assert abs(float(lse[t, h]) - math.log(den)) < 1e-12
    none, z, _ = orc.attention(q, codes, scales, table, [0, 2], [6], 0.3, end=[0, 0])
    assert (none == 0).all() and (z == float("-inf")).all()


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4, 30, generator=g, dtype=torch.float64) * 2
    x[1, :20] = float("-inf")
    x[3] = float("-inf")
    tok = torch.tensor([3, 25, -1, 2])
    gl, gh = torch.randn(4, generator=g, dtype=torch.float64), torch.randn(4, generator=g, dtype=torch.float64)
    grad = orc.token_logprobs_backward(x, tok, 0.7, gl, gh)

    def value(y):
        lp, h = orc.token_logprobs(y, tok, 0, 0.7)[:2]
        return float((gl[:3] * lp[:3] + gh[:3] * h[:3]).sum())

    for r in range(3):
        for i in range(30):
            if x[r, i] == float("-inf"):
                assert grad[r, i] == 0
                continue
            d = torch.zeros_like(x)
            d[r, i] = 1e-5
            assert abs((value(x + d) - value(x - d)) / 2e-5 - float(grad[r, i])) < 1e-8
    assert (grad[3] == 0).all()


def test_order_of_alternatives():
    nan, inf = float("nan"), float("inf")
    assert orc.ordered(torch.tensor([1.0, nan, -0.0, 0.0, 1.0, -inf, inf])) == [6, 0, 4, 2, 3, 5, 1]
