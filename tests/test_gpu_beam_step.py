"""The beam-search step under grammars against the CPU oracle (masks, states) and the plain selection, and the
example that runs the step together with the paged cache."""
import os
import sys

import numpy as np
import pytest
import torch

import beam_ref as ref
import oracle
from test_gpu_beam import TOL, as_dtype
from wg_workloads import flatten, grammars, has_structural_byte, make_vocab

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


class Search:
    """A search on the library beside the same one on the oracle: cursors instead of states."""

    def __init__(self, wg, vocab, ops, R, K, *, capacity=4096, mode=None, flags=0, norm=0, dtype="fp32"):
        self.wg, self.vocab, self.R, self.K, self.norm, self.flags, self.dtype = wg, vocab, R, K, norm, flags, dtype
        n = R * K
        flats = [flatten(op) for op in ops]
        self.trees, self.grammars = [oracle.Tree(f) for f in flats], [wg.Grammar(f) for f in flats]
        self.dv = wg.Vocab(vocab.offsets, vocab.data, vocab.eos_id)
        self.ctx = wg.Context(self.dv, capacity, n, **({} if mode is None else {"cache_mode": mode}))
        ids = [self.ctx.add_grammar(g) for g in self.grammars]
        self.which = [r % len(ops) for r in range(R) for _ in range(K)]         # each row's grammar
        self.ids = ids
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.gid, self.sid = i32([ids[w] for w in self.which]), i32([self.grammars[w].start_state for w in self.which])
        self.cursors = [self.trees[w].start() for w in self.which]
        self.score = np.where(np.arange(n) % K == 0, 0, -np.inf).astype(np.float32)
        self.d_score = torch.from_numpy(self.score).cuda()
        self.mask = torch.zeros((n, self.dv.W), dtype=torch.int32, device="cuda")
        self.parent, self.token, self.status = i32([0] * n), i32([0] * n), i32([9] * n)
        self.beam = wg.Beam(vocab.size, R, K)
        self.empty = 0

    def step(self, logits):
        """logits: CPU tensor [rows, V]."""
        n, K, V = self.R * self.K, self.K, self.vocab.size
        words = oracle.masks([self.trees[w] for w in self.which], self.vocab, self.cursors)
        allowed = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :V].astype(bool)
        finished = [c == oracle.DONE for c in self.cursors]
        want = ref.select(logits.float().numpy(), allowed, self.score, finished, self.vocab.eos_id, self.norm, self.R, K)
        self.wg.wg_beam_step(self.beam, self.ctx, K, self.gid, self.sid, self.d_score, logits.cuda(), self.mask, self.parent,
                             self.token, self.status, norm=self.norm, flags=self.flags)
        torch.cuda.synchronize()
        parent, token, score = self.parent.cpu().numpy(), self.token.cpu().numpy(), self.d_score.cpu().numpy()
        status = self.status.cpu().numpy()
        cursors, which = list(self.cursors), list(self.which)
        for r, line in enumerate(want):
            for j in range(K):
                i = r * K + j
                if j >= len(line):
                    assert parent[i] == -1 and token[i] == -1 and score[i] == -np.inf and status[i] == self.wg.WG_ERR_EMPTY_MASK
                    self.empty += 1
                    continue
                s, b, t = line[j]
                assert (parent[i], token[i], status[i]) == (b, t, 0), (i, line[j], parent[i], token[i], score[i])
                assert abs(score[i] - s) <= TOL
                which[i] = self.which[r * K + b]
                rc, cursors[i] = oracle.advance(self.trees[which[i]], self.vocab, self.cursors[r * K + b], t)
                assert rc == 0
        self.cursors, self.which, self.score = cursors, which, score
        assert self.gid.tolist() == [self.ids[w] for w in which]
        return parent, token

    def check_states(self):
        """Every row's device state allows exactly what its oracle cursor allows."""
        out = torch.zeros_like(self.mask)
        self.wg.wg_build_masks(self.ctx, self.gid, self.sid, out, self.wg.WG_NO_CACHE)
        want = oracle.masks([self.trees[w] for w in self.which], self.vocab, self.cursors)
        assert (out.cpu().numpy().view(np.uint32) == want).all()


@pytest.fixture(scope="module")
def vocab():
    return make_vocab(2500, seed=3)


OPS = [lambda: grammars.json_reference_lookup(doc_nodes=40), lambda: grammars.html_template(), lambda: grammars.random_template(seed=5)]


@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("R,K,kind", [(1, 1, "dense"), (3, 4, "dense"), (3, 4, "compact"), (2, 8, "none"), (4, 5, "tiny"), (30, 3, "dense")])
def test_search(wg, vocab, R, K, kind, norm):
    """dense / compact cache, no cache, and a cache that takes three masks (the rest is built every step)."""
    s = Search(wg, vocab, [op() for op in OPS], R, K, norm=norm, capacity={"tiny": 3}.get(kind, 4096),
               mode=wg.WG_CACHE_COMPACT if kind == "compact" else None, flags=wg.WG_NO_CACHE if kind == "none" else 0)
    rng = np.random.default_rng(R * 10 + K + norm)
    bonus = 6.0 * has_structural_byte(vocab).astype(np.float32)
    for step in range(14):
        s.step(as_dtype(rng.standard_normal((R * K, vocab.size)) * 2 + bonus, "fp32"))
        if step % 5 == 4:
            s.check_states()
    s.check_states()
    assert s.ctx.stats()["empty_masks"] == s.empty and s.ctx.stats()["bad_states"] == 0


@pytest.mark.parametrize("R,K,kind", [(150, 2, "dense"), (150, 2, "compact"), (10, 32, "dense"), (20, 32, "compact")])
def test_search_of_many_requests(wg, vocab, R, K, kind):
    """Batches on both sides of what one launch takes."""
    s = Search(wg, vocab, [op() for op in OPS], R, K, mode=wg.WG_CACHE_COMPACT if kind == "compact" else None)
    rng = np.random.default_rng(R + K)
    bonus = 6.0 * has_structural_byte(vocab).astype(np.float32)
    for _ in range(4):
        s.step(as_dtype(rng.standard_normal((R * K, vocab.size)) * 2 + bonus, "fp32"))
    s.check_states()


def test_search_to_the_end(wg):
    """A language of a few short words: beams finish, keep their scores, and there are fewer words than beams."""
    vocab = make_vocab(600, seed=9)
    words = wg.RegexTree(r"[ab]x")
    tree = oracle.Tree(words)
    g = wg.Grammar.from_regex(r"[ab]x")
    dv = wg.Vocab(vocab.offsets, vocab.data, vocab.eos_id)
    K = 5
    ctx = wg.Context(dv, 64, K)
    gid = torch.full((K,), ctx.add_grammar(g), dtype=torch.int32, device="cuda")
    sid = torch.full((K,), g.start_state, dtype=torch.int32, device="cuda")
    score = torch.tensor([0.0] + [-np.inf] * (K - 1), device="cuda")
    mask = torch.zeros((K, dv.W), dtype=torch.int32, device="cuda")
    beam = wg.Beam(vocab.size, 1, K)
    steps = 5
    token, parent = (torch.zeros((steps, 1, K), dtype=torch.int32, device="cuda") for _ in range(2))
    logits = torch.randn((K, vocab.size), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    for i in range(steps):
        wg.wg_beam_step(beam, ctx, K, gid, sid, score, logits, mask, parent[i].view(-1), token[i].view(-1))
    out = torch.zeros((1, K, steps), dtype=torch.int32, device="cuda")
    wg.wg_beam_backtrack(token, parent, out)
    live = score > -np.inf
    texts = [b"".join(vocab.token(t) for t in line if t != vocab.eos_id) for line in out[0][live].tolist()]
    assert live.any() and set(texts) <= {b"ax", b"bx"} and {b"ax", b"bx"} <= set(texts)
    assert (sid[live] == g.done_state).all() and (out[0][~live] == -1).all()
    assert torch.equal(score, score.sort(descending=True).values)
    for text in texts:
        assert tree.accepts(list(text) + [256])


def test_step_refusals(wg, vocab):
    s = Search(wg, vocab, [OPS[1]()], 2, 4)
    x = torch.zeros((8, vocab.size), device="cuda")
    call = lambda **k: wg.wg_beam_step(**dict(dict(beam=s.beam, ctx=s.ctx, n_beam=4, gid=s.gid, sid=s.sid, score=s.d_score, logits=x,  # noqa: E731
                                                   bitmask=s.mask, parent_out=s.parent, token_out=s.token), **k))
    call()
    small = wg.Context(s.dv, 16, 7)
    small.add_grammar(s.grammars[0])
    other = wg.Beam(vocab.size + 1, 2, 4)
    for error, k in ((ValueError, dict(n_beam=3)), (wg.WgError, dict(ctx=small)), (wg.WgError, dict(beam=other)), (wg.WgError, dict(flags=2)),
                     (wg.WgError, dict(norm=5)), (ValueError, dict(gid=s.gid[:7])), (ValueError, dict(score=s.d_score[:7])),
                     (TypeError, dict(score=s.gid)), (ValueError, dict(token_out=None)), (ValueError, dict(parent_out=None)),
                     (ValueError, dict(bitmask=s.mask[:, :-1])), (ValueError, dict(logits=x[:, :-1])), (wg.WgError, dict(n_beam=8))):
        with pytest.raises(error):
            call(**k)
    # masks cached for a slice of the vocabulary only are not taken for whole ones
    big = make_vocab(20000, seed=4)
    dv = wg.Vocab(big.offsets, big.data, big.eos_id)
    ctx = wg.Context(dv, 64, 8)
    gid = torch.full((8,), ctx.add_grammar(s.grammars[0]), dtype=torch.int32, device="cuda")
    sid = torch.full((8,), s.grammars[0].start_state, dtype=torch.int32, device="cuda")
    mask = torch.zeros((8, dv.W), dtype=torch.int32, device="cuda")
    keys = torch.zeros(8, dtype=torch.int64, device="cuda")
    wg.wg_decode_step_shard(ctx, gid, sid, torch.zeros((8, 8192), device="cuda"), mask, 0, 8192, keys)
    args = (wg.Beam(20000, 2, 4), ctx, 4, gid, sid, s.d_score, torch.zeros((8, 20000), device="cuda"), mask, s.parent, s.token)
    with pytest.raises(wg.WgError):
        wg.wg_beam_step(*args)
    ctx.cache_clear()
    wg.wg_beam_step(*args)
    torch.cuda.synchronize()


def test_unknown_states_end_a_beam(wg, vocab):
    """A grammar or state id that the context does not have: no candidates, counted, nothing faults."""
    s = Search(wg, vocab, [OPS[1]()], 2, 2)
    s.d_score.zero_()
    s.gid[0], s.sid[2] = 77, 1 << 20
    s.gid[1] = -3
    x = torch.randn((4, vocab.size), device="cuda")
    wg.wg_beam_step(s.beam, s.ctx, 2, s.gid, s.sid, s.d_score, x, s.mask, s.parent, s.token, s.status)
    # (what is left of the second request: beam 1 in the grammar's start state)
    n = min(2, int(np.unpackbits(oracle.masks(s.trees, vocab, [s.trees[0].start()]).view(np.uint8)).sum()))
    assert n > 0 and s.parent.tolist() == [-1, -1] + [1] * n + [-1] * (2 - n)
    assert s.status.tolist() == [-6, -6] + [0] * n + [-6] * (2 - n)
    assert s.gid.tolist()[:2] == [77, -3] and s.ctx.stats()["bad_states"] == 3


def test_example_against_a_dense_cache(wg):
    """The example's search on the paged cache and on a cache that is copied whole at every step."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import beam_search as ex

    class DenseCache:
        def __init__(self, rows, most):
            self.keys, self.values = (torch.zeros((rows, -(-most // ex.BLOCK) * ex.BLOCK, ex.DIM), device="cuda") for _ in range(2))
            self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")

        def append(self, n_new, tokens, model):
            k, v = model.keys_values(tokens)
            at = 0
            for row, n in enumerate(n_new.tolist()):
                p = int(self.lens[row])
                self.keys[row, p:p + n], self.values[row, p:p + n] = k[at:at + n], v[at:at + n]
                at += n
            self.lens += n_new

        def read(self):
            return self.keys, self.values

        def follow(self, parent):
            R, K = parent.shape
            row = (torch.arange(R, device="cuda")[:, None] * K + parent.clamp(min=0)).view(-1)
            self.keys, self.values = self.keys[row], self.values[row]
            self.lens = torch.where(parent.view(-1) < 0, 0, self.lens[row]).to(torch.int32)

    vocab = make_vocab(2000, seed=1)
    grammar = wg.Grammar(flatten(grammars.json_reference_lookup(doc_nodes=30)))
    model = ex.ToyModel(vocab)
    prompts = [[11, 12, 13], list(range(40, 61))]
    steps, K = 40, 4
    paged = ex.search(model, vocab, grammar, prompts, K, steps)
    dense = ex.search(model, vocab, grammar, prompts, K, steps, DenseCache(2 * K, 21 + steps + 1))
    assert torch.equal(paged[0], dense[0]) and torch.equal(paged[2], dense[2])
    assert torch.allclose(paged[1], dense[1], rtol=1e-4, atol=1e-3)
    assert (paged[0] >= 0).any()
