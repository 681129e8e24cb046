"""Greedy decoding through one sparse-attention layer, from the library's calls:

    paged_plan        pages and slots of the step's tokens
    cache4_append     their keys and values, in 4 bits
    indexer_topk      the keys that each token is to read
    cache4_attention  attention over those (or, for the prompt, over all)
    token_logprobs    what the logits say of the chosen token

The model is one layer with random weights; what matters is how the calls hang
together. Sequences lie one after the other in the indexer's key array, `room`
positions each, so its lists hold positions of that array; cache4_attention takes
each sequence's start off them again (selected_start).

    python examples/decode_step.py
"""
from __future__ import annotations

import os
import sys
from types import SimpleNamespace

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_11976_amd import litetopk as lt  # noqa: E402

HEADS, KV_HEADS, DIM = 8, 2, 64     # attention
INDEX_HEADS, INDEX_DIM = 4, 64      # indexer
WIDTH, VOCAB = 256, 4096
PAGE = 16


def weights(seed: int = 0) -> SimpleNamespace:
    g = torch.Generator(device="cuda").manual_seed(seed)

    def mat(rows, cols):
        return torch.randn(rows, cols, generator=g, device="cuda") / rows ** 0.5

    return SimpleNamespace(embed=torch.randn(VOCAB, WIDTH, generator=g, device="cuda"), q=mat(WIDTH, HEADS * DIM),
                           k=mat(WIDTH, KV_HEADS * DIM), v=mat(WIDTH, KV_HEADS * DIM), o=mat(HEADS * DIM, WIDTH),
                           iq=mat(WIDTH, INDEX_HEADS * INDEX_DIM), ik=mat(WIDTH, INDEX_DIM),
                           iw=mat(WIDTH, INDEX_HEADS), head=mat(WIDTH, VOCAB))


class Decoder:
    """The state of a batch of sequences: 4-bit pages, indexer keys, lengths."""

    def __init__(self, w: SimpleNamespace, sequences: int, room: int, selected: int):
        self.w, self.n, self.room, self.selected = w, sequences, room, selected
        per = (room + PAGE - 1) // PAGE
        self.codes, self.scales = lt.cache4_empty(sequences * per, PAGE, KV_HEADS, DIM)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((sequences, per), -1, **i32)
        self.free = torch.randperm(sequences * per, device="cuda").int()
        self.used = torch.zeros(1, **i32)
        self.lens = torch.zeros(sequences, **i32)
        self.index_keys = torch.zeros(sequences * room, INDEX_DIM, device="cuda")
        self.starts = torch.arange(sequences, **i32) * room

    def step(self, tokens: torch.Tensor, new_lens: torch.Tensor, sparse: bool):
        """Logits after the last token of each sequence; tokens lie in sequence order."""
        w, x = self.w, self.w.embed[tokens]
        plan = lt.paged_plan(self.lens, new_lens, self.table, self.free, self.used, PAGE, tokens.numel())
        if plan.status.any():
            raise RuntimeError("no room for the new tokens of sequences %s" % plan.status.nonzero().flatten().tolist())
        lt.cache4_append((x @ w.k).view(-1, KV_HEADS, DIM), (x @ w.v).view(-1, KV_HEADS, DIM), self.codes, self.scales,
                         plan.slots)
        seq = torch.repeat_interleave(torch.arange(self.n, device="cuda"), new_lens)
        start = self.starts[seq]
        self.index_keys[(start + plan.positions).long()] = x @ w.ik
        picked = None
        if sparse:
            picked, _ = lt.indexer_topk((x @ w.iq).view(-1, INDEX_HEADS, INDEX_DIM), torch.relu(x @ w.iw),
                                        self.index_keys, self.selected, start + plan.positions + 1,
                                        options=lt.make_options(visible_start=start))
        out, _ = lt.cache4_attention((x @ w.q).view(-1, HEADS, DIM).to(torch.bfloat16), self.codes, self.scales,
                                     self.table, plan.cu_tokens, plan.seq_lens, selected=picked,
                                     selected_start=start if sparse else None)
        self.lens, self.used = plan.seq_lens, plan.free_used
        y = x + out.float().flatten(1) @ w.o
        return y[(plan.cu_tokens[1:] - 1).long()] @ w.head


def generate(prompts, steps: int, selected: int = 32, sparse: bool = True, seed: int = 0):
    """(tokens, log probabilities, entropies) [sequences, steps] of greedy decoding."""
    lens = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device="cuda")
    room = max(len(p) for p in prompts) + steps
    dec = Decoder(weights(seed), len(prompts), room, selected)
    logits = dec.step(torch.tensor([t for p in prompts for t in p], device="cuda"), lens, sparse=False)
    one = torch.ones_like(lens)
    tokens, logprobs, entropies = [], [], []
    for _ in range(steps):
        # the best alternative of the row is the token that comes next
        best = lt.token_logprobs(logits, torch.full((len(prompts),), -1, device="cuda"), top=1)
        tokens.append(best.top_index[:, 0].long())
        logprobs.append(best.top_logprob[:, 0])
        entropies.append(best.entropy)
        logits = dec.step(tokens[-1], one, sparse)
    return torch.stack(tokens, 1), torch.stack(logprobs, 1), torch.stack(entropies, 1)


def main():
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, VOCAB, (n,), generator=g).tolist() for n in (40, 7, 133)]
    tokens, logprobs, entropies = generate(prompts, steps=12)
    for r in range(len(prompts)):
        print("sequence %d: tokens %s, mean log probability %.3f, mean entropy %.3f"
              % (r, tokens[r].tolist(), logprobs[r].mean(), entropies[r].mean()))


if __name__ == "__main__":
    main()
