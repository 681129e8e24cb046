"""GPU: rows of a paged cache that go on as their parents, against the plain
definition, and over many steps of a search whose beams' histories are known."""
import random

import pytest
import torch

from oracle import serving_oracle as orc
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _run(table, lens, parents, group, page, free, used, keep=None, width=None):
    rows = len(lens)
    t = _int(table).view(rows, -1) if rows else torch.zeros(0, width or 0, dtype=torch.int32, device="cuda")
    f = _int(free)
    r = lt.paged_reorder(t, _int(lens), _int(parents), group, f, _int([used]), page,
                         keep_pages=None if keep is None else _int(keep))
    return dict(block_table=r.block_table.tolist(), seq_lens=r.seq_lens.tolist(), copies=r.copies.tolist(),
                free_used=r.free_used.tolist(), status=r.status.tolist(), free=f.tolist())


def _tree(reqs, group, page, width, seed, spare, idle=0.1):
    """Tables as beam search leaves them: rows share pages up to where they parted."""
    rng = random.Random(seed)
    table, lens, pages = [], [], 0
    for _ in range(reqs):
        n = rng.randint(0, width * page)
        first = rng.randint(0, n // page)
        mine = []
        for w in range(group):
            m = 0 if rng.random() < idle else max(0, min(width * page, n + rng.randint(-2, 2)))
            count = -(-m // page)
            row = []
            if mine:
                source, length = rng.choice(mine)
                row = source[:min(rng.randint(first, max(first, n // page)), count, length // page)]
            row = row + list(range(pages, pages + count - len(row)))
            pages += sum(1 for p in row if p >= pages)
            mine.append((row, m))
            table.append(row + [-1] * (width - count))
            lens.append(m)
    order = list(range(pages + spare))
    rng.shuffle(order)
    table = [[order[p] if p >= 0 else -1 for p in row] for row in table]
    used = order[:pages]
    rng.shuffle(used)
    return table, lens, used + order[pages:], pages, rng


@pytest.mark.parametrize("reqs,group,page,width,spare", [
    (1, 1, 16, 5, 3), (1, 4, 16, 9, 0), (5, 3, 1, 7, 4), (9, 8, 64, 33, 20), (2, 64, 16, 130, 0), (3, 33, 4, 65, 9),
    (40, 16, 16, 70, 100), (7, 5, 128, 1, 1), (1, 64, 16, 700, 3), (2, 2, 16, 2000, 3)])
@pytest.mark.parametrize("few", [False, True])
def test_matches_definition(lib, reqs, group, page, width, spare, few):
    for seed in range(4):
        table, lens, free, used, rng = _tree(reqs, group, page, width, 10 * seed + few, spare)
        # parents: any, or a few that take all
        pick = [rng.randrange(group) for _ in range(2)] if few else list(range(-1, group + 1))
        parents = [rng.choice(pick) for _ in lens]
        keep = [rng.randint(0, 2)] * len(lens) if seed == 3 else None
        want = orc.paged_reorder(table, lens, parents, group, page, free, used, keep)
        got = _run(table, lens, parents, group, page, free, used, keep)
        for name in want:
            assert got[name] == want[name], (seed, name)


@pytest.mark.parametrize("reqs,group", [(1, 15), (15, 1), (4, 4), (2, 8), (1, 16), (17, 1), (1, 17), (6, 3), (31, 1), (2, 16),
                                        (8, 4), (33, 1)])
@pytest.mark.parametrize("page,width", [(16, 63), (4, 513)])
def test_rows_of_one_launch_and_of_two(lib, reqs, group, page, width):
    for seed in range(2):
        table, lens, free, used, rng = _tree(reqs, group, page, width, 100 + seed, 7)
        parents = [rng.choice(list(range(-1, group)) + [0, 0]) for _ in lens]
        want = orc.paged_reorder(table, lens, parents, group, page, free, used)
        got = _run(table, lens, parents, group, page, free, used)
        for name in want:
            assert got[name] == want[name], (seed, name)


def test_no_pages_left(lib):
    # prompts in the first row of each group; all rows go on as it: copies beyond the list end
    group, page, width = 4, 16, 3
    table = [[2 * (r // group), 2 * (r // group) + 1, -1] if r % group == 0 else [-1] * 3 for r in range(8)]
    lens = [20 if r % group == 0 else 0 for r in range(8)]
    for total in range(4, 11):
        want = orc.paged_reorder(table, lens, [0] * 8, group, page, list(range(total)), 4)
        got = _run(table, lens, [0] * 8, group, page, list(range(total)), 4)
        assert got == want and want["status"].count(2) == max(0, 10 - total)


def test_odd_inputs(lib):
    """Lengths beyond the table, negative ones, entries that are no page, parents that are none, a mark outside the list."""
    table = [[5, 6], [5, 7], [8, -1], [-1, -1]]
    for lens in ([1000, 40, 17, -5], [32, 31, 30, 1], [0x7FFFFFFF, -1, 16, 0]):
        for parents in ([0, 0, 1, 1], [3, 3, 3, 3], [-7, 99, 2, 2], [2, 1, 0, 0]):
            for used in (9, 0, -3, 1000, 2):
                free = list(range(12))
                want = orc.paged_reorder(table, lens, parents, 4, 16, free, used)
                assert _run(table, lens, parents, 4, 16, free, used) == want
    r = _run([], [], [], 4, 16, [1, 2], 1, width=3)
    assert r["free_used"] == [1] and r["block_table"] == []


def test_strided_table_and_most_rows(lib):
    rows, group, page, width = lt.LT_PLAN_MAX_REQUESTS, 8, 16, 3
    table, lens, free, used, rng = _tree(rows // group, group, page, width, 5, 10)
    parents = [rng.randrange(-1, group) for _ in lens]
    want = orc.paged_reorder(table[:800], lens[:800], parents[:800], group, page, free, used)
    got = _run(table[:800], lens[:800], parents[:800], group, page, free, used)
    assert got == want
    # all rows, in a wider table: those that need no page of the list are known row by row
    wide = torch.full((rows, 7), -9, dtype=torch.int32, device="cuda")
    wide[:, 2:5] = _int(table)
    f = _int(free)
    r = lt.paged_reorder(wide[:, 2:5], _int(lens), _int(parents), group, f, _int([used]), page)
    lens_t, go = torch.tensor(lens), torch.tensor(parents) >= 0
    at = torch.arange(rows) // group * group + torch.tensor(parents).clamp(min=0)
    good = r.status.cpu() == 0
    assert torch.equal(good | (r.status.cpu() == 2), go)
    assert torch.equal(r.seq_lens.cpu(), torch.where(good, lens_t[at], 0).int())
    plain = good & (r.copies[:, 0].cpu() < 0)
    held = (lens_t[at] + page - 1) // page
    rowed = torch.tensor(table)[at]
    rowed = torch.where(torch.arange(width) < held[:, None], rowed, -1)
    assert torch.equal(r.block_table.cpu()[plain], rowed.int()[plain])
    # pages in use and on the list: none twice
    used2 = int(r.free_used)
    live = {p for row in r.block_table.tolist() for p in row if p >= 0}
    assert live.isdisjoint(f[used2:].tolist()) and len(set(f[used2:].tolist())) == len(f[used2:])
    assert torch.all(wide[:, :2] == -9) and torch.all(wide[:, 5:] == -9)


def test_copies_of_pages(lib):
    for heads, d, page, pages in [(8, 128, 64, 9), (1, 64, 1, 9), (3, 64, 16, 9), (2, 128, 1, 9), (5, 128, 128, 9)]:
        g = torch.Generator(device="cuda").manual_seed(1)
        codes = torch.randint(0, 256, (pages, heads, page, 2, d // 2), generator=g, device="cuda", dtype=torch.uint8)
        scales = torch.randint(0, 256, (pages, heads, page, 2, d // 32), generator=g, device="cuda", dtype=torch.uint8)
        a, b = codes.clone(), scales.clone()
        lt.cache4_copy(codes, scales, _int([[2, 7], [-1, -1], [2, 0], [3, 99], [99, 4], [-1, 5], [5, -1], [8, 1], [6, 6]]))
        a[[7, 0, 1]], b[[7, 0, 1]] = a[[2, 2, 8]], b[[2, 2, 8]]
        assert torch.equal(codes, a) and torch.equal(scales, b)


def test_histories_of_a_search(lib):
    """Beams grow and part at random over 40 steps; every row's cache holds its own history's tokens."""
    rng = random.Random(7)
    group, reqs, page, width, heads, d = 4, 3, 4, 14, 2, 64
    rows, total = group * reqs, 120
    codes, scales = lt.cache4_empty(total, page, heads, d)
    table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
    lens, used = torch.zeros(rows, dtype=torch.int32, device="cuda"), _int([0])
    free = torch.randperm(total, generator=torch.Generator().manual_seed(8)).int().cuda()
    histories = [[] for _ in range(rows)]

    def key(tokens):  # a token's key and value: a code per value, exact in 4 bits
        n = torch.tensor(tokens, device="cuda")[:, None, None]
        v = ((n >> (torch.arange(heads * d, device="cuda").view(heads, d) % 12)) & 1).float()
        return v + 1.0, 3.0 - v

    made = 0
    for step in range(40):
        new = [rng.randint(1, 6) if step == 0 and r % group == 0 else int(bool(histories[r])) for r in range(rows)]
        plan = lt.paged_plan(lens, _int(new), table, free, used, page, sum(new))
        assert not plan.status.any()
        tokens = []
        for r in range(rows):
            fresh = list(range(made, made + new[r]))
            made += new[r]
            histories[r] = histories[r] + fresh
            tokens += fresh
        k, v = key(tokens)
        lt.cache4_append(k, v, codes, scales, plan.slots)
        pick = [[w for w in range(group) if histories[g * group + w]] for g in range(reqs)]
        parents = [rng.choice(pick[r // group]) for r in range(rows)]
        r = lt.paged_reorder(table, plan.seq_lens, _int(parents), group, free, plan.free_used, page)
        lt.cache4_copy(codes, scales, r.copies)
        assert not r.status.any()
        table, lens, used = r.block_table, r.seq_lens, r.free_used
        histories = [list(histories[i // group * group + parents[i]]) for i in range(rows)]
        assert lens.tolist() == [len(h) for h in histories]
        for i in range(rows):
            at = torch.arange(len(histories[i]), device="cuda")
            slots = table[i, at // page].long() * page + at % page
            got = lt.cache4_read(codes, scales, slots)
            want = key(histories[i])
            assert torch.equal(got[0].float(), want[0]) and torch.equal(got[1].float(), want[1])
    assert used.item() < total // 2


def test_argument_errors_raise(lib):
    t, v = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    f, u = torch.arange(9, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = [lambda: lt.paged_reorder(t.cpu(), v, v.clone(), 4, f, u, 16), lambda: lt.paged_reorder(t, v, v.long(), 4, f, u, 16),
             lambda: lt.paged_reorder(t, v, v[:2], 4, f, u, 16), lambda: lt.paged_reorder(t, v, v, 3, f, u, 16),
             lambda: lt.paged_reorder(t, v, v, 0, f, u, 16), lambda: lt.paged_reorder(t, v, v, 4, f, u, 15),
             lambda: lt.paged_reorder(t[:3], v, v, 4, f, u, 16), lambda: lt.paged_reorder(t.t(), v[:3], v[:3], 3, f, u, 16),
             lambda: lt.paged_reorder(t, v, v, 4, f, f, 16), lambda: lt.paged_reorder(t, v, v, 4, f.cpu(), u, 16),
             lambda: lt.paged_reorder(t, v, v, 4, f, u, 16, workspace=torch.zeros(8, dtype=torch.uint8, device="cuda"))]
    c, s = lt.cache4_empty(2, 16, 1, 64)
    calls += [lambda: lt.cache4_copy(c, s, v), lambda: lt.cache4_copy(c, s, t), lambda: lt.cache4_copy(c, s, t[:, :2]),
              lambda: lt.cache4_copy(c, s, t[:, :2].contiguous().cpu()), lambda: lt.cache4_copy(c, s, torch.zeros(2, 2))]
    for i, call in enumerate(calls):
        with pytest.raises(lt.LiteTopKError):
            call()
            print("call %d was taken" % i)
