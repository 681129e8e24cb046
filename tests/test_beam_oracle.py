"""The plain definitions of rotary positions, beam selection and reordered pages,
pinned by hand and by what they have to keep."""
import itertools
import math
import random

import pytest
import torch

from oracle import serving_oracle as orc


def test_rotary_by_hand():
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    f = torch.tensor([math.pi / 2])
    half = orc.rotary(x, torch.tensor([1]), f, start=1)
    assert torch.allclose(half, torch.tensor([[[1.0, -3.0, 2.0, 4.0, 5.0]]], dtype=torch.float64), atol=1e-6)
    both = orc.rotary(x, torch.tensor([1]), torch.tensor([math.pi / 2, math.pi]), start=1, amplitude=2.0)
    # pairs (1, 3) by a quarter, (2, 4) by a half turn
    assert torch.allclose(both, torch.tensor([[[1.0, -8.0, -6.0, 4.0, -10.0]]], dtype=torch.float64), atol=1e-5)
    inter = orc.rotary(x, torch.tensor([1]), torch.tensor([math.pi / 2, math.pi]), interleaved=True)
    assert torch.allclose(inter, torch.tensor([[[-2.0, 1.0, -3.0, -4.0, 5.0]]], dtype=torch.float64), atol=1e-5)
    assert torch.equal(orc.rotary(x, torch.tensor([-1]), f), torch.zeros(1, 1, 5, dtype=torch.float64))


def test_rotary_keeps_lengths_and_turns_back():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 3, 12, generator=g)
    pos = torch.tensor([0, 1, 77, 1 << 20, 5])
    f = torch.rand(5, generator=g)
    for inter in (False, True):
        y = orc.rotary(x, pos, f, 1, inter)
        assert torch.allclose(y.square().sum(-1), x.double().square().sum(-1))
        assert torch.allclose(orc.rotary(y, pos, f, 1, inter, inverse=True), x.double())
        assert torch.equal(y[0], x[0].double())


def test_rotary_scores_depend_on_distances():
    g = torch.Generator().manual_seed(2)
    q, k = torch.randn(1, 1, 8, generator=g), torch.randn(1, 1, 8, generator=g)
    f = torch.rand(4, generator=g)

    def score(a, b):
        return (orc.rotary(q, torch.tensor([a]), f) * orc.rotary(k, torch.tensor([b]), f)).sum()

    assert abs(score(9, 4) - score(1005, 1000)) < 1e-9


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0001, 1), (447.9, 0), (224.0, -1), (1.75, -8), (1.76, -7), (0.0, -126),
                                   (1e-45, -126), (3e38, 120)])
def test_fp8_exponent(top, e):
    assert orc.fp8_exponent(top) == e


def test_beam_scores_by_hand():
    x = torch.tensor([[0.0, math.log(3.0)], [5.0, -math.inf], [1.0, math.nan], [2.0, math.inf], [-math.inf, -math.inf],
                      [7.0, 7.0]])
    cum = torch.tensor([[-1.0, -2.0, 0.0, 0.0, 0.0, -math.inf]])
    y = orc.beam_scores(x, cum)
    want = [[math.log(0.25) - 1, math.log(0.75) - 1], [-2.0, -math.inf]] + [[-math.inf, -math.inf]] * 4
    assert torch.allclose(y, torch.tensor([want], dtype=torch.float64))


@pytest.mark.parametrize("low", [-1e30, torch.finfo(torch.float32).min, torch.finfo(torch.bfloat16).min, 1e30])
def test_beam_scores_of_far_rows(low):
    """Where a row lies does not matter: equal values share the probability, however large they are."""
    x = torch.tensor([[low] * 4, [low] * 2 + [-math.inf] * 2, [2.0 * low if low < -1e38 else -abs(low)] * 4], dtype=torch.float64)
    cum = torch.tensor([[-3.0, -1.0, -2.0]])
    y = orc.beam_scores(x, cum)[0]
    want = [[-3.0 - math.log(4)] * 4, [-1.0 - math.log(2)] * 2 + [-math.inf] * 2, [-2.0 - math.log(4)] * 4]
    assert torch.allclose(y, torch.tensor(want, dtype=torch.float64), rtol=0, atol=1e-12)


def test_reorder_by_hand():
    # two rows share page 4; row 0 has 5, row 1 has 6; three tokens a... page of 2: lengths 3
    table, lens = [[4, 5, -1], [4, 6, -1]], [3, 3]
    r = orc.paged_reorder(table, lens, [0, 0], 2, 2, [5, 4, 6, 7], 3)
    # row 1 ended: page 6 goes back, and is what the second child's copy takes
    assert r["block_table"] == [[4, 5, -1], [4, 6, -1]] and r["copies"] == [[-1, -1], [5, 6]]
    assert r["free"] == [5, 4, 6, 7] and r["free_used"] == [3] and r["status"] == [0, 0]
    r = orc.paged_reorder(table, lens, [1, -1], 2, 2, [5, 4, 6, 7], 3)
    assert r["block_table"] == [[4, 6, -1], [-1] * 3] and r["free"] == [5, 4, 5, 7] and r["free_used"] == [2]
    assert r["status"] == [0, 1] and r["seq_lens"] == [3, 0]
    # both end: the shared page goes back once
    r = orc.paged_reorder(table, lens, [-1, 2], 2, 2, [5, 4, 6, 7], 3)
    assert r["free"][:3] == [6, 5, 4] and r["free_used"] == [0]
    # all go on as row 0, whose length is even: nothing to copy
    r = orc.paged_reorder(table, [2, 3], [0, 0], 2, 2, [5, 4, 6, 7], 3)
    assert r["copies"] == [[-1, -1]] * 2 and r["block_table"] == [[4, -1, -1]] * 2
    # no page left for the copy
    r = orc.paged_reorder([[0, -1], [-1, -1]], [1, 0], [0, 0], 2, 2, [0], 1)
    assert r["status"] == [0, 2] and r["seq_lens"] == [1, 0] and r["block_table"] == [[0, -1], [-1, -1]]


def test_reorder_keeps_count_of_pages():
    """Over many steps of beams that grow and part: pages in use and pages on the list are all there are."""
    rng = random.Random(3)
    group, reqs, page, width, total = 4, 3, 2, 12, 200
    rows = group * reqs
    table, lens = [[-1] * width for _ in range(rows)], [0] * rows
    free, used = list(range(total)), 0
    for step in range(20):
        new = [1 if (lens[r] or r % group == 0) else 0 for r in range(rows)]
        plan = orc.paged_plan(lens, new, table, free, used, page, rows)
        assert not any(plan["status"])
        table, lens, used = plan["table"], plan["seq_lens"], plan["free_used"][0]
        parents = [rng.choice([w for w in range(group) if lens[g * group + w]])
                   for g, _ in itertools.product(range(reqs), range(group))]
        r = orc.paged_reorder(table, lens, parents, group, page, free, used)
        table, lens, free, used = r["block_table"], r["seq_lens"], r["free"], r["free_used"][0]
        in_use = {p for row, n in zip(table, lens) for p in row[:-(-n // page)]}
        assert in_use.isdisjoint(free[used:]) and len(in_use) == used and len(set(free[used:])) == total - used
