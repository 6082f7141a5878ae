"""Beam-search steps queued one behind the other, without a synchronisation, with the beams of a request in
different grammars: the grammar ids that a step writes are those the next call on them reads.

The whole search is first run on the oracle, which also makes the logits.  Candidates next to each other in a
request's order are kept at least GAP apart, so that the order does not hang on roundings: scores stay
below 256 in size, so each of the two roundings of a step is at most 2^-17 and the logarithm of the sum is good
to 2^-16 + 2^-16 (exponent and its own rounding); 21 steps are off by at most 21 * 3 * 2^-16 = 2^-10.
"""
import numpy as np
import pytest
import torch

import beam_ref as ref
import oracle
from test_gpu_beam import as_dtype
from test_gpu_beam_step import OPS, Search
from wg_workloads import make_vocab

pytestmark = pytest.mark.gpu
STEPS = 20
GAP = 2.0 ** -8


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


@pytest.fixture(scope="module")
def vocab():
    return make_vocab(2500, seed=3)


class Mixed(Search):
    """A search whose beams begin in different grammars, all of them alive."""

    def __init__(self, wg, vocab, R, K, **k):
        super().__init__(wg, vocab, [op() for op in OPS], R, K, **k)
        self.which = [(i % K + i // K) % len(OPS) for i in range(R * K)]
        self.cursors = [self.trees[w].start() for w in self.which]
        self.score = -3 * np.random.default_rng(R + K).random(R * K)
        self.gid.copy_(torch.tensor([self.ids[w] for w in self.which], dtype=torch.int32))
        self.sid.copy_(torch.tensor([self.grammars[w].start_state for w in self.which], dtype=torch.int32))
        self.score = self.score.astype(np.float32).astype(np.float64)
        self.d_score.copy_(torch.from_numpy(self.score))

    def allowed(self):
        words = oracle.masks([self.trees[w] for w in self.which], self.vocab, self.cursors)
        return np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :self.vocab.size].astype(bool)

    def logits(self, rng, rows, allowed):
        """One likely token per row, with log-probabilities that let the rows overtake each other: all rows live on
        and change places."""
        x = np.full((len(rows), self.vocab.size), -60.0, np.float32)
        for i, row in enumerate(rows):
            tokens = np.flatnonzero(allowed[row])
            tokens = tokens[tokens != self.vocab.eos_id] if len(tokens) > 1 else tokens
            if len(tokens):
                x[i, rng.choice(tokens)] = -3 * rng.random()
        return as_dtype(x, self.dtype)

    def plan(self, rng):
        """One step of the oracle: its logits, parents and tokens; -1 where no candidate is left."""
        R, K, n = self.R, self.K, self.R * self.K
        allowed, finished = self.allowed(), [c == oracle.DONE for c in self.cursors]
        x = self.logits(rng, range(n), allowed)
        best = [None] * R
        again = list(range(R))
        for _ in range(200):
            rows = [r * K + b for r in again for b in range(K)]
            lines = ref.select(x[rows].float().numpy(), allowed[rows], self.score[rows], [finished[i] for i in rows],
                               self.vocab.eos_id, self.norm, len(again), K + 1)
            for r, line in zip(again, lines):
                best[r] = line
            # (candidates at -60 and below stay behind in any order)
            again = [r for r in again if any(a[0] - b[0] < GAP and a[0] > -55 for a, b in zip(best[r], best[r][1:]))]
            if not again:
                break
            rows = [r * K + b for r in again for b in range(K)]
            x[rows] = self.logits(rng, rows, allowed)
        assert not again
        parent, token = (np.full(n, -1, np.int32) for _ in range(2))
        cursors, which, score = list(self.cursors), list(self.which), np.full(n, -np.inf)
        for r, line in enumerate(best):
            line = [c for c in line[:K] if c[0] > -55]
            assert len(line) == min(K, sum(self.score[r * K:(r + 1) * K] > -np.inf) - self.stuck(allowed, finished, r))
            for j, (s, b, t) in enumerate(line):
                i, p = r * K + j, r * K + b
                parent[i], token[i], which[i], score[i] = b, t, self.which[p], s
                rc, cursors[i] = oracle.advance(self.trees[which[i]], self.vocab, self.cursors[p], t)
                assert rc == 0
        assert (np.abs(score[score > -np.inf]) < 256).all()
        self.cursors, self.which, self.score = cursors, which, score
        return x, parent, token

    def stuck(self, allowed, finished, r):
        rows = range(r * self.K, (r + 1) * self.K)
        return sum(1 for i in rows if self.score[i] > -np.inf and not finished[i] and not allowed[i].any())


@pytest.mark.parametrize("dtype,norm", [("fp32", ref.NORM_NONE), ("bf16", ref.NORM_NONE)])
@pytest.mark.parametrize("R,K", [(2, 4), (40, 6), (200, 2), (170, 8)])
@pytest.mark.parametrize("between", ["nothing", "reorder", "graph"])
def test_steps_queued_back_to_back(wg, vocab, R, K, dtype, norm, between):
    """Both sides of what one launch takes; by themselves, with the cache's tables moved in between, and
    recorded.  A greedy step and its advance follow at once."""
    s = Mixed(wg, vocab, R, K, norm=norm, dtype=dtype)
    n = R * K
    start = s.gid.clone(), s.sid.clone(), s.d_score.clone()
    rng = np.random.default_rng(R * 10 + K)
    xs, parents, tokens, moved = [], [], [], 0
    for _ in range(STEPS):
        before = list(s.which)
        x, p, t = s.plan(rng)
        moved += sum(a != b for a, b in zip(before, s.which))
        xs.append(x), parents.append(p), tokens.append(t)
    assert moved > n                       # grammar ids really move
    # what a greedy step on the last states has to choose: the lowest token of the largest allowed logit
    last = as_dtype(rng.standard_normal((n, vocab.size)), dtype)
    allowed = s.allowed()
    greedy = np.where(allowed.any(1), np.where(allowed, last.float().numpy(), -np.inf).argmax(1), -1)
    d_xs = [x.cuda() for x in xs]
    d_last = last.cuda()
    d_parent, d_token = (torch.full((STEPS, n), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    d_greedy = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    tables = plain = None
    if between == "reorder":
        plain = ref.Tables(3 * n, 4, n, 6)
        lens = np.full(n, 9)               # two full blocks and a partly filled one
        plain.extend([int(v) for v in lens], int(lens.sum()))
        pool = wg.KvPool(3 * n, 4, n)
        table = torch.from_numpy(plain.table()).cuda()
        d_lens = torch.from_numpy(lens.astype(np.int32)).cuda()
        pool.load(torch.from_numpy(np.array(plain.ref, np.int32)).cuda())
        tables = wg.KvTables(pool, table, d_lens)

    def queue():
        for i in range(STEPS):
            wg.wg_beam_step(s.beam, s.ctx, K, s.gid, s.sid, s.d_score, d_xs[i], s.mask, d_parent[i], d_token[i], s.status,
                            norm=norm)
            if tables is not None:
                tables.reorder(d_parent[i].view(R, K))
        wg.wg_decode_step(s.ctx, s.gid, s.sid, d_last, s.mask, d_greedy)

    if between == "graph":
        graph = torch.cuda.CUDAGraph()
        queue()                            # (kernels are loaded before they are recorded)
        d_last.copy_(last)
        for to, was in zip((s.gid, s.sid, s.d_score), start):
            to.copy_(was)
        d_parent.fill_(-7), d_token.fill_(-7)
        with torch.cuda.graph(graph):
            queue()
        graph.replay()
    else:
        torch.cuda.synchronize()
        queue()
    torch.cuda.synchronize()
    assert (d_parent.cpu().numpy() == np.stack(parents)).all()
    assert (d_token.cpu().numpy() == np.stack(tokens)).all()
    assert s.gid.tolist() == [s.ids[w] for w in s.which]
    assert (d_greedy.cpu().numpy() == greedy).all()
    for i, t in enumerate(greedy):
        if t >= 0:
            rc, s.cursors[i] = oracle.advance(s.trees[s.which[i]], vocab, s.cursors[i], int(t))
            assert rc == 0
    s.check_states()
    if plain is not None:
        for p in parents:
            plain.reorder(p.reshape(R, K))
        assert (table.cpu().numpy() == plain.table()).all() and d_lens.tolist() == plain.len
