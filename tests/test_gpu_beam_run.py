"""GPU: the calls of a beam search together, as a program makes them: a search through
the paged cache against the same sequences decoded alone, on given streams, and captured
into a graph that is replayed beside eager work."""
import math

import pytest
import torch

from examples import decode_step as ex
from paper_2607_11976_amd import litetopk as lt

pytestmark = pytest.mark.gpu


def _prompts(lens=(21, 5, 40)):
    g = torch.Generator().manual_seed(3)
    return [torch.randint(0, ex.VOCAB, (n,), generator=g).tolist() for n in lens]


def test_a_search_scores_its_sequences_as_they_score_alone(lib):
    """Every finished beam's score is the sum of its tokens' log probabilities when the sequence
    is decoded by itself, without beams or shared pages. The keys that both cache are the same bit
    for bit (rotation and codes depend on the token alone); attention sums them in other shares,
    each output off by 2^-8 of itself as bfloat16 at most, which moves logits of size 3 by 3 * 2^-8
    over a hidden state half of which is attention: 0.05 a step is several times that."""
    beams, steps = 4, 9
    prompts = _prompts()
    tokens, scores = ex.beam_search(prompts, beams, steps)
    assert tokens.shape == (len(prompts), beams, steps) and torch.all(scores[:, :-1] >= scores[:, 1:])
    for r, prompt in enumerate(prompts):
        assert len({tuple(t) for t in tokens[r].tolist()}) == beams
        for b in range(beams):
            alone = ex.score_alone(prompt, tokens[r, b].tolist())
            assert abs(alone - scores[r, b].item()) < 0.05 * steps, (r, b)


def test_one_beam_is_greedy(lib):
    """A search with one beam takes the best token at each step."""
    prompts = _prompts((13, 30))
    tokens, scores = ex.beam_search(prompts, 1, 6)
    again, same = ex.beam_search(prompts, 1, 6)
    assert torch.equal(tokens, again) and torch.equal(scores, same)
    for r, prompt in enumerate(prompts):
        dec = ex.BeamDecoder(ex.weights(0), 1, 1, len(prompt) + 6)
        logits = dec.step(torch.tensor(prompt, device="cuda"), torch.tensor([len(prompt)], dtype=torch.int32, device="cuda"))
        assert logits.argmax(-1).item() == tokens[r, 0, 0].item()


def test_one_beam_is_greedy_at_every_step(lib):
    """Decoded on with the search's own tokens, in the same batch and without selecting or reordering rows, every
    step's best logit is the token that the search took next, and its score is the sum of their log probabilities:
    each step adds the log sum's error and rounds a score of this size once."""
    prompts, steps = _prompts((13, 30)), 6
    tokens, scores = ex.beam_search(prompts, 1, steps)
    dec = ex.BeamDecoder(ex.weights(0), len(prompts), 1, max(len(p) for p in prompts) + steps)
    logits, one = dec.prompt(prompts), torch.ones(len(prompts), dtype=torch.int32, device="cuda")
    total = torch.zeros(len(prompts), dtype=torch.float64, device="cuda")
    for i in range(steps):
        assert torch.equal(logits.argmax(-1), tokens[:, 0, i])
        total += torch.log_softmax(logits.double(), -1).amax(-1)
        logits = dec.step(tokens[:, 0, i], one)
    slack = (2 * math.log(ex.VOCAB) + 2 * (ex.VOCAB // 1024 + 41) + 10) * 2.0 ** -24    # as in test_log_sums
    assert torch.all((scores[:, 0].double() - total).abs() <= steps * (slack + 2.0 ** -24 * total.abs()))


def test_pages_come_back(lib):
    """Beams that are given up return their pages: after a long search as many are in use as the
    surviving rows hold."""
    beams, steps = 4, 25
    dec = ex.BeamDecoder(ex.weights(0), 2, beams, 64 + steps)
    g = torch.Generator().manual_seed(5)
    total = dec.free.numel()
    dec.prompt(_prompts((17, 9)))
    for _ in range(steps):
        parents = torch.randint(0, beams, (2 * beams,), generator=g).int().cuda()
        dec.go_on(parents)
        dec.step(torch.randint(0, ex.VOCAB, (2 * beams,), generator=g).cuda(), torch.ones(2 * beams, dtype=torch.int32, device="cuda"))
        rows = [row[:-(-n // ex.PAGE)] for row, n in zip(dec.table.tolist(), dec.lens.tolist())]
        held = {p for row in rows for p in row}
        assert min(held) >= 0 and len(held) == dec.used.item() < total
        assert held.isdisjoint(dec.free[dec.used.item():].tolist())


def _step(s, stream=None):
    """One step of a search of 3 requests with 4 beams, from buffers that stay in place."""
    kw = {} if stream is None else {"stream": stream}
    with torch.cuda.stream(stream):
        for to, what in zip((s.codes, s.scales, s.free), s.first):
            to.copy_(what)
    plan = lt.paged_plan(s.lens, s.new, s.table, s.free, s.used, 16, 12, **kw)
    q = lt.cache4_append_rotary(s.k, s.v, s.codes, s.scales, plan.slots, plan.positions, s.rot, q=s.q, **kw)
    out, lse = lt.cache4_attention(q, s.codes, s.scales, s.table, plan.cu_tokens, plan.seq_lens, **kw)
    picked = lt.beam_select(s.logits, s.scores, 8, **kw)
    r = lt.paged_reorder(s.table, plan.seq_lens, s.parents, 4, s.free, plan.free_used, 16, **kw)
    lt.cache4_copy(s.codes, s.scales, r.copies, **kw)
    ix = lt.rotary_fp8(s.q, plan.positions, s.rot, **kw)
    back = lt.rotary_backward(s.q, plan.positions, s.rot, **kw)
    return [q, out, lse, *picked, *r, *ix, back]


class _State:
    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def rand(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        i32 = dict(dtype=torch.int32, device="cuda")
        self.rot = lt.rotary_frequencies(64)
        self.q, self.k, self.v = (rand(12, h, 64).to(torch.bfloat16) for h in (8, 2, 2))
        self.logits, self.scores = rand(12, 5000) * 3, rand(3, 4)
        self.codes, self.scales = lt.cache4_empty(80, 16, 2, 64)
        lt.cache4_append(rand(1280, 2, 64), rand(1280, 2, 64), self.codes, self.scales, torch.arange(1280, device="cuda"))
        self.table = torch.full((12, 6), -1, **i32)
        self.table[:, :3] = torch.randperm(36, generator=g, device="cuda").view(12, 3)
        self.lens, self.new = torch.full((12,), 40, **i32), torch.ones(12, **i32)
        self.free, self.used = torch.arange(80, **i32), torch.full((1,), 36, **i32)
        self.parents = torch.randint(0, 4, (12,), generator=g, device="cuda").int()
        # what a step writes is put back before the next: copies go to pages given back, which rows
        # without children still name in this table
        self.first = [t.clone() for t in (self.codes, self.scales, self.free)]

    def values(self):
        return [self.codes, self.scales, self.free, self.table]


def _same(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert x.dtype == y.dtype and x.shape == y.shape
        x, y = (t.view(torch.uint8) if t.element_size() == 1 else t for t in (x, y))
        assert torch.equal(torch.nan_to_num(x) if x.is_floating_point() else x,
                           torch.nan_to_num(y) if y.is_floating_point() else y)


def test_on_a_given_stream(lib):
    s, t = _State(1), _State(1)
    want = _step(s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = _step(t, side)
    torch.cuda.current_stream().wait_stream(side)
    _same(got, want)
    _same(t.values(), s.values())


def test_captured_and_replayed(lib):
    """A graph of the step, replayed with eager steps of another state in between, and two graphs of
    their own memory replayed in turn: each replay gives what an eager step gives."""
    s, other = _State(2), _State(3)
    want, want_other = _step(_State(2)), _step(_State(3))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(s)
        _step(other)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for state in (s, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = _step(state)
        graphs.append((graph, got))
    for _ in range(4):
        for t in graphs[0][1] + graphs[1][1]:
            t.zero_() if t.element_size() > 1 else t.view(torch.uint8).zero_()
        graphs[0][0].replay()
        eager = _step(_State(3))
        graphs[1][0].replay()
        torch.cuda.synchronize()
        _same(graphs[0][1], want)
        _same(graphs[1][1], want_other)
        _same(eager, want_other)


def test_captured_selection_follows_its_inputs(lib):
    """A captured selection reads the logits and scores that are there when it is replayed: other
    beams alive, other values."""
    x, cum = torch.zeros(8, 40000, device="cuda"), torch.zeros(2, 4, device="cuda")
    lt.beam_select(x, cum, 6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lt.beam_select(x, cum, 6)
    g = torch.Generator(device="cuda").manual_seed(9)
    for alive in (4, 1, 2, 0, 3):
        x.copy_(torch.randn(8, 40000, generator=g, device="cuda"))
        cum.copy_(torch.where(torch.arange(4, device="cuda") < alive, -torch.rand(2, 4, generator=g, device="cuda"), -math.inf))
        graph.replay()
        _same(list(got), list(lt.beam_select(x.clone(), cum.clone(), 6)))
