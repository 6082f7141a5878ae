"""The forms in which a search is run in earnest: 16-bit logits over a full-size vocabulary, rows at odd places, steps queued over a
cache that has no room, other streams, recorded calls."""
import numpy as np
import pytest
import torch

import beam_ref as ref
import oracle
from test_gpu_beam import TOL, as_dtype
from test_gpu_beam_queued import STEPS, Mixed
from test_gpu_beam_step import OPS, Search
from test_gpu_kv import Both, i32
from wg_workloads import has_structural_byte, make_vocab

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def draw(s, rng, bonus):
    """Logits for the search's next step: no two of a request's K + 1 best candidates of different beams lie within 2 * TOL."""
    R, K, V = s.R, s.K, s.vocab.size
    words = oracle.masks([s.trees[w] for w in s.which], s.vocab, s.cursors)
    allowed = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :V].astype(bool)
    finished = [c == oracle.DONE for c in s.cursors]
    new = lambda rows: as_dtype(rng.standard_normal((len(rows), V)) * 2 + bonus, s.dtype)  # noqa: E731
    x = new(range(R * K))
    again = list(range(R))
    for _ in range(60):
        rows = [r * K + b for r in again for b in range(K)]
        xf = x[rows].float().numpy()
        lines = ref.select(xf, allowed[rows], s.score[rows], [finished[i] for i in rows], s.vocab.eos_id, s.norm, len(again), K + 1)
        close = []
        for at, (r, line) in enumerate(zip(again, lines)):
            for (s0, b0, t0), (s1, b1, t1) in zip(line, line[1:]):
                if s0 - s1 < 2 * TOL and (b0 != b1 or xf[at * K + b0, t0] != xf[at * K + b1, t1]):
                    close.append(r)
        again = sorted(set(close))
        if not again:
            return x
        rows = [r * K + b for r in again for b in range(K)]
        x[rows] = new(rows)
    raise AssertionError("no separated logits found")


SMALL = [(2501, 3, 4, "dense"), (2501, 160, 3, "compact"), (2503, 2, 5, "none")]
LARGE = [(128256, 1, 4, "dense"), (128259, 2, 8, "compact")]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,R,K,kind,norm", [(*size, norm) for size in SMALL for norm in (0, 1, 2)] + [(*size, norm) for size in LARGE for norm in (0, 1)])
def test_search_in_both_types(wg, V, R, K, kind, dtype, norm):
    """Odd vocabularies: every row begins elsewhere in a piece of 16 bytes.  One launch and two."""
    vocab = make_vocab(V, seed=3)
    s = Search(wg, vocab, [op() for op in OPS], R, K, norm=norm, dtype=dtype,
               mode=wg.WG_CACHE_COMPACT if kind == "compact" else None, flags=wg.WG_NO_CACHE if kind == "none" else 0)
    rng = np.random.default_rng(V + R + norm)
    bonus = 6.0 * has_structural_byte(vocab).astype(np.float32)
    for _ in range(4 if V > 100000 else 8):
        s.step(draw(s, rng, bonus))
    s.check_states()


@pytest.mark.parametrize("kind", ["tiny", "compact", "none"])
@pytest.mark.parametrize("R,K", [(30, 4), (200, 2)])
def test_queued_steps_without_room_in_the_cache(wg, R, K, kind):
    """Masks that are built anew at every step, into rows that the step before has read: nothing stale is seen."""
    vocab = make_vocab(2500, seed=3)
    s = Mixed(wg, vocab, R, K, norm=ref.NORM_NONE, dtype="bf16", capacity=3 if kind == "tiny" else 4096,
              mode=wg.WG_CACHE_COMPACT if kind == "compact" else None, flags=wg.WG_NO_CACHE if kind == "none" else 0)
    rng = np.random.default_rng(R + K)
    plans = [s.plan(rng) for _ in range(STEPS)]
    xs = [x.cuda() for x, _, _ in plans]
    parent, token = (torch.full((STEPS, R * K), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    for i in range(STEPS):
        wg.wg_beam_step(s.beam, s.ctx, K, s.gid, s.sid, s.d_score, xs[i], s.mask, parent[i], token[i], norm=s.norm, flags=s.flags)
    torch.cuda.synchronize()
    assert (parent.cpu().numpy() == np.stack([p for _, p, _ in plans])).all()
    assert (token.cpu().numpy() == np.stack([t for _, _, t in plans])).all()
    s.check_states()


def test_a_step_on_another_stream(wg):
    vocab = make_vocab(2500, seed=3)
    s = Search(wg, vocab, [op() for op in OPS], 3, 4)
    rng = np.random.default_rng(0)
    bonus = 6.0 * has_structural_byte(vocab).astype(np.float32)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                # the current stream is taken
        for _ in range(4):
            s.step(draw(s, rng, bonus))
    side.synchronize()
    # and a stream that is named: it is busy for a while, so work on any other would come too early
    x = draw(s, rng, bonus)
    src, late = x.cuda(), torch.full_like(x, -1.0, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        late.copy_(src)
    wg.wg_beam_step(s.beam, s.ctx, 4, s.gid, s.sid, s.d_score, late, s.mask, s.parent, s.token, stream=side)
    side.synchronize()
    got = s.parent.tolist(), s.token.tolist()
    words = oracle.masks([s.trees[w] for w in s.which], vocab, s.cursors)
    allowed = np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :vocab.size].astype(bool)
    want = ref.select(x.numpy(), allowed, s.score, [c == oracle.DONE for c in s.cursors], vocab.eos_id, 0, 3, 4)
    pad = lambda line, at: [c[at] for c in line] + [-1] * (4 - len(line))  # noqa: E731
    assert got == ([b for line in want for b in pad(line, 1)], [t for line in want for t in pad(line, 2)])


def tables_round(both, slots, new, parent, keep, planes, stream=None):
    """A step's calls on the tables: room for tokens, the selection followed, drafted tokens given back."""
    both.tables.extend(new, slots, stream=stream)
    both.tables.reorder(parent, planes, stream=stream)
    both.tables.shrink(keep, stream=stream)


@pytest.mark.parametrize("how", ["graph", "stream"])
def test_tables_recorded_and_on_another_stream(wg, how):
    R, K, block = 5, 6, 4
    n = R * K
    both = Both(wg, n * 12, block, n, 12)
    planes = [torch.randn((n * 12, block, 8), device="cuda"), torch.randint(0, 99, (n * 12, block, 3), device="cuda", dtype=torch.uint8)]
    rng = np.random.default_rng(5)
    both.extend(rng.integers(1, 10, n), 10 * n)
    # (grown by two and cut to a fixed length that all reach in the end: every round finds other lengths)
    new, parent, keep = np.full(n, 2), rng.integers(0, K, (R, K)), np.full(n, 9)
    d_new, d_parent, d_keep = i32(new), i32(parent), i32(keep)
    slots = wg.SlotMap(n, 2 * n)
    d_planes = wg.KvPlanes(planes, block)
    want = [p.clone() for p in planes]
    torch.cuda.synchronize()
    if how == "graph":
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            tables_round(both, slots, d_new, d_parent, d_keep, d_planes)
        go = graph.replay
    else:
        side = torch.cuda.Stream()
        go = lambda: tables_round(both, slots, d_new, d_parent, d_keep, d_planes, stream=side)  # noqa: E731
    for _ in range(4):
        go()
    torch.cuda.synchronize()
    for _ in range(4):
        cu, slot, pos, seq, _ = both.plain.extend([2] * n, 2 * n)
        copies, _, _, _ = both.plain.reorder(parent)
        for p in want:
            for a, b, tokens in copies:
                p[b, :tokens] = p[a, :tokens]
        both.plain.shrink([9] * n)
    both.same()
    for got, w in zip((slots.cu, slots.slot, slots.pos, slots.seq), (cu, slot, pos, seq)):
        assert (got.cpu().numpy() == w).all()
    assert all(torch.equal(p, w) for p, w in zip(planes, want))


@pytest.mark.parametrize("T,R,K", [(40, 5, 3), (4500, 3, 8)])
def test_backtrack_recorded_and_on_another_stream(wg, T, R, K):
    rng = np.random.default_rng(T)
    token = rng.integers(0, 1 << 20, (T, R, K)).astype(np.int32)
    parent = rng.integers(0, K, (T, R, K)).astype(np.int32)
    parent[rng.random((T, R, K)) < 0.2 / T] = -1
    want = ref.backtrack(token, parent)
    d_token, d_parent = (torch.zeros((T, R, K), dtype=torch.int32, device="cuda") for _ in range(2))
    out = torch.zeros((R, K, T), dtype=torch.int32, device="cuda")
    wg.wg_beam_backtrack(d_token, d_parent, out)
    src = torch.from_numpy(token).cuda(), torch.from_numpy(parent).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                # (busy for a while: a call on another stream would come too early)
        torch.cuda._sleep(20_000_000)
        d_token.copy_(src[0]), d_parent.copy_(src[1])
    wg.wg_beam_backtrack(d_token, d_parent, out, stream=side)
    side.synchronize()
    assert (out.cpu().numpy() == want).all()
    out.fill_(-9)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        wg.wg_beam_backtrack(d_token, d_parent, out)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert (out.cpu().numpy() == want).all()
