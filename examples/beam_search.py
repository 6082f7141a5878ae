"""Beam search under a grammar, with a paged key / value cache.

A toy language model (one attention layer, random weights, synthetic vocabulary) fills in a JSON
reference lookup.  The model's part is plain PyTorch, its attention too unless ``--storage`` says what the library's
is to hold; what the library does is everything around it:

  KvTables.extend      cache slots for the step's tokens (block tables from lengths, on the GPU)
  wg_beam_step         masks of the beams' automaton states, selection, states of the chosen beams
  KvTables.reorder     the block tables follow the selection; shared blocks stay shared
  wg_beam_backtrack    the hypotheses read back
  KvCache.write        with --storage: keys and queries rotated, keys and values quantised into their slots
  Attend               and the attention over them, a request's prompt read once for all of its beams

    python examples/beam_search.py [--requests 2] [--beams 4] [--steps 48] [--storage bf16|e4m3|int8]
"""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2507_16768_b200 as wg  # noqa: E402
from wg_workloads import flatten, grammars, has_structural_byte, make_vocab  # noqa: E402

DIM, BLOCK = 64, 16


class ToyModel:
    """logits = head(embedding + attention over the sequence so far)."""

    def __init__(self, vocab, seed: int = 0, steer: float = 4.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *n: torch.randn(n, device="cuda", generator=g) / DIM ** 0.5  # noqa: E731
        self.embed, self.k, self.v, self.head = rand(vocab.size, DIM) * 4, rand(DIM, DIM), rand(DIM, DIM), rand(DIM, vocab.size) * 4
        # tokens with structural characters are made likelier, so that free text ends
        self.bias = steer * torch.from_numpy(has_structural_byte(vocab).astype(np.float32)).cuda()

    def keys_values(self, tokens):
        e = self.embed[tokens]
        return e @ self.k, e @ self.v

    def logits(self, tokens, keys, values, lens):
        """tokens [rows]; keys, values [rows, positions, DIM], of which the first lens[rows] count."""
        e = self.embed[tokens]
        w = (keys @ e[:, :, None])[:, :, 0]
        w = torch.where(torch.arange(w.shape[1], device=w.device)[None, :] < lens[:, None], w, -1e30)
        w = torch.softmax(w, 1)
        return self.output(tokens, (w[:, :, None] * values).sum(1))

    def output(self, tokens, context):
        return (self.embed[tokens] + context) @ self.head + self.bias


class PagedCache:
    """Keys and values in blocks; rows of requests x beams."""

    def __init__(self, rows: int, most: int, n_blocks: int):
        blocks = -(-most // BLOCK)
        self.pool = wg.KvPool(n_blocks, BLOCK, rows)
        self.table = torch.full((rows, blocks), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.tables = wg.KvTables(self.pool, self.table, self.lens, self.status)
        self.keys, self.values = (torch.zeros((n_blocks, BLOCK, DIM), device="cuda") for _ in range(2))
        self.planes = wg.KvPlanes([self.keys, self.values], BLOCK)
        self.at = torch.arange(blocks * BLOCK, device="cuda")

    def append(self, n_new, tokens, model):
        """tokens: those of all rows one after the other, n_new[row] for each."""
        slots = wg.SlotMap(n_new.numel(), tokens.numel())
        self.tables.extend(n_new, slots)
        k, v = model.keys_values(tokens)
        ok = slots.slot >= 0
        self.keys.view(-1, DIM)[slots.slot[ok]] = k[ok]
        self.values.view(-1, DIM)[slots.slot[ok]] = v[ok]

    def read(self):
        slot = self.table.clamp(min=0)[:, self.at // BLOCK].long() * BLOCK + self.at % BLOCK
        return self.keys.view(-1, DIM)[slot], self.values.view(-1, DIM)[slot]

    def follow(self, parent):
        self.tables.reorder(parent, self.planes)


class LibraryCache(PagedCache):
    """The same with the library's cache and attention: one head, 16-bit queries, what is held in 16 or 8 bits."""

    def __init__(self, rows: int, most: int, n_blocks: int, n_beam: int, storage: str = "bf16"):
        super().__init__(rows, most, n_blocks)
        held = {"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[storage]
        self.cache = wg.KvCache.empty(n_blocks, BLOCK, 1, DIM, held)
        self.planes = self.cache.planes
        self.rope, self.attention, self.n_beam = wg.Rope(most, DIM), wg.Attend(rows, 1, 1, DIM), n_beam
        self.queries = torch.zeros((rows, 1, DIM), dtype=torch.bfloat16, device="cuda")

    def append(self, n_new, tokens, model):
        slots = wg.SlotMap(n_new.numel(), tokens.numel())
        self.tables.extend(n_new, slots)
        k, v = (x.to(torch.bfloat16)[:, None] for x in model.keys_values(tokens))
        q = model.embed[tokens].to(torch.bfloat16)[:, None].contiguous()
        self.cache.write(k, v, slots, rope=self.rope, q=q)
        last = (slots.cu[1:] - 1).long().clamp(min=0)        # of every row's new tokens
        self.queries = torch.where((n_new > 0)[:, None, None], q[last], self.queries) if tokens.numel() else self.queries

    def attend(self):
        out = torch.empty_like(self.queries)
        self.attention(self.queries, self.cache, self.tables, out, scale=1.0, group=self.n_beam)
        return out[:, 0].float()


def search(model, vocab, grammar, prompts, n_beam: int, steps: int, cache=None):
    """Returns (tokens [requests, beams, steps], scores [requests, beams], finished [requests, beams])."""
    R, rows = len(prompts), len(prompts) * n_beam
    most = max(len(p) for p in prompts) + steps + 1
    if cache is None:
        cache = PagedCache(rows, most, rows * (-(-most // BLOCK) + 1))
    dev_vocab = wg.Vocab(vocab.offsets, vocab.data, vocab.eos_id)
    ctx = wg.Context(dev_vocab, cache_capacity=4096, max_batch=rows)
    beam = wg.Beam(vocab.size, R, n_beam)
    new = lambda dtype, value=0, shape=(rows,): torch.full(shape, value, dtype=dtype, device="cuda")  # noqa: E731
    gid = new(torch.int32, ctx.add_grammar(grammar))
    sid = new(torch.int32, grammar.start_state)
    bitmask = new(torch.int32, 0, (rows, dev_vocab.W))
    score = new(torch.float32, -float("inf")).view(R, n_beam)
    score[:, 0] = 0.0                                   # one hypothesis per request at first
    score = score.reshape(-1).contiguous()
    token_steps = new(torch.int32, 0, (steps, R, n_beam))
    parent_steps = new(torch.int32, 0, (steps, R, n_beam))
    # the prompts go into the first beams; their last tokens are what the first step works on
    last = new(torch.int64)
    n_new = new(torch.int32)
    for r, p in enumerate(prompts):
        last[r * n_beam:(r + 1) * n_beam] = p[-1]
        n_new[r * n_beam] = len(p)
    cache.append(n_new, torch.tensor([t for p in prompts for t in p], device="cuda"), model)
    for step in range(steps):
        if isinstance(cache, LibraryCache):
            logits = model.output(last, cache.attend())
        else:
            keys, values = cache.read()
            logits = model.logits(last, keys, values, cache.lens)
        parent, token = parent_steps[step].view(-1), token_steps[step].view(-1)
        wg.wg_beam_step(beam, ctx, n_beam, gid, sid, score, logits, bitmask, parent, token)
        cache.follow(parent.view(R, n_beam))
        running = (score > -float("inf")) & (token != vocab.eos_id)
        last = token.clamp(min=0).long()
        tokens = torch.where(running, last, 0)
        cache.append(running.to(torch.int32), tokens[running], model)
    out = new(torch.int32, 0, (R, n_beam, steps))
    wg.wg_beam_backtrack(token_steps, parent_steps, out)
    return out, score.view(R, n_beam), (sid == grammar.done_state).view(R, n_beam)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=2)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--steps", type=int, default=48)
    ap.add_argument("--storage", choices=("bf16", "e4m3", "int8"), help="attention by the library, over a cache of this")
    a = ap.parse_args()
    vocab = make_vocab(32000, seed=1)
    grammar = wg.Grammar(flatten(grammars.json_reference_lookup(doc_nodes=60)))
    model = ToyModel(vocab)
    prompts = [[10 + 7 * r + i for i in range(5 + 9 * r)] for r in range(a.requests)]
    cache = None
    if a.storage:
        rows, most = a.requests * a.beams, max(len(p) for p in prompts) + a.steps + 1
        cache = LibraryCache(rows, most, rows * (-(-most // BLOCK) + 1), a.beams, a.storage)
    out, score, finished = search(model, vocab, grammar, prompts, a.beams, a.steps, cache)
    for r in range(a.requests):
        for j in range(a.beams):
            text = b"".join(vocab.token(t) for t in out[r, j].tolist() if t >= 0 and t != vocab.eos_id)
            print(f"request {r} beam {j}: {score[r, j].item():9.3f} {'finished' if finished[r, j] else 'running ':8s} {text!r}")


if __name__ == "__main__":
    main()
