"""Constrained beam search on the GPU against a plain implementation in 64 bits.

Tolerance of a score, derived before the first run: the kernel forms lse in fp32 and rounds twice,
fl(score + fl(x - lse)).  With |score|, |x|, |lse| <= M every rounding is at most M * 2^-23, the sum of up
to 2^18 positive terms and its exponentials (2 ulp each, arguments exact to one rounding scaled by at
most 60) are together good to 2^-16 relative, which is an absolute 2^-16 in the logarithm.  So
|error| <= 2^-16 + 4 * M * 2^-23; M = 64 covers the inputs here: 4.6e-5.

Which candidates are chosen is compared exactly; the inputs keep candidates of different beams further
apart than twice that tolerance (or exactly equal in both arithmetics, where order goes by index).
"""
import numpy as np
import pytest
import torch

import beam_ref as ref

pytestmark = pytest.mark.gpu
TOL = 2.0 ** -16 + 4 * 64 * 2.0 ** -23


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def as_dtype(x, dtype):
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32))
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def run(wg, logits, allowed, score, finished, eos, norm, n_req, n_out, offset=0, pad=0, beam=None):
    """One wg_beam_select on `logits` (CPU tensor [rows, V]) laid out with rows `V + pad` apart and
    beginning `offset` elements into their allocation."""
    rows, V = logits.shape
    K = rows // n_req
    store = torch.full((offset + rows * (V + pad),), float("nan"), dtype=logits.dtype, device="cuda")
    view = torch.as_strided(store, (rows, V), (V + pad, 1), offset)
    view.copy_(logits.cuda())
    mask = None if allowed is None else torch.from_numpy(ref.pack_mask(allowed).view(np.int32)).cuda()
    out = (torch.zeros((n_req, n_out), dtype=torch.float32, device="cuda"),
           torch.zeros((n_req, n_out), dtype=torch.int32, device="cuda"),
           torch.zeros((n_req, n_out), dtype=torch.int32, device="cuda"))
    if beam is None:
        beam = wg.Beam(V, n_req, K, n_out)
    fin = None if finished is None else torch.from_numpy(np.ascontiguousarray(finished, np.int32)).cuda()
    wg.wg_beam_select(beam, K, view, torch.from_numpy(np.ascontiguousarray(score, np.float32)).cuda(), *out, bitmask=mask,
                      finished=fin, eos_id=eos, norm=norm)
    torch.cuda.synchronize()
    return tuple(o.cpu().numpy() for o in out)


def check(got, want, tol=TOL):
    score, parent, token = got
    for r, line in enumerate(want):
        n = len(line)
        assert parent[r, :n].tolist() == [b for _, b, _ in line], (r, score[r], line)
        assert token[r, :n].tolist() == [t for _, _, t in line], (r, score[r], line)
        np.testing.assert_allclose(score[r, :n], [s for s, _, _ in line], rtol=0, atol=tol)
        assert (parent[r, n:] == -1).all() and (token[r, n:] == -1).all() and np.isneginf(score[r, n:]).all()


def separate(x, allowed, score, finished, eos, norm, n_req, n_out, rng):
    """Scores for which no two of the n_out + 1 best candidates of different beams lie within 2 * TOL."""
    K = len(x) // n_req
    for _ in range(50):
        close = []
        for r, line in enumerate(ref.select(x, allowed, score, finished, eos, norm, n_req, n_out + 1)):
            for (s0, b0, t0), (s1, b1, t1) in zip(line, line[1:]):
                if s0 - s1 < 2 * TOL and (b0 != b1 or x[r * K + b0, t0] != x[r * K + b1, t1]):
                    close.append(r)
        if not close:
            return score
        for r in set(close):
            live = score[r * K:(r + 1) * K] > -np.inf
            score[r * K:(r + 1) * K][live] = -10 * rng.random(int(live.sum()), dtype=np.float32)
    raise AssertionError("no separated scores found")


def make(seed, n_req, K, V, dtype, kind, norm, n_out, dead=True):
    rng = np.random.default_rng(seed)
    rows = n_req * K
    x = as_dtype(np.round(rng.standard_normal((rows, V)) * 2 * 1024) / 1024, dtype)
    xf = x.float().numpy()
    allowed = {"all": lambda: np.ones((rows, V), bool),
               "most": lambda: rng.random((rows, V)) < 0.93,
               "few": lambda: rng.random((rows, V)) < 12 / V,
               "one": lambda: np.arange(V)[None, :] == rng.integers(0, V, (rows, 1)),
               "none": lambda: np.zeros((rows, V), bool)}[kind]()
    if kind == "few" and rows > 2:
        allowed[1] = False
    score = -10 * rng.random(rows, dtype=np.float32)
    finished = (rng.random(rows) < 0.15) if dead else np.zeros(rows, bool)
    if dead and rows > 1:
        score[rng.random(rows) < 0.1] = -np.inf
    eos = int(rng.integers(0, V))
    score = separate(xf, allowed, score, finished, eos, norm, n_req, n_out, rng)
    return x, xf, allowed, score, finished, eos


@pytest.mark.parametrize("norm", [ref.NORM_ALLOWED, ref.NORM_FULL, ref.NORM_NONE])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["all", "most", "few", "one", "none"])
@pytest.mark.parametrize("n_req,K,V,n_out", [
    (1, 1, 1, 1), (1, 1, 31, 4), (2, 3, 257, 3), (3, 4, 1023, 8), (2, 2, 1025, 5), (1, 5, 4099, 64), (4, 8, 9000, 16)])
def test_selection(wg, n_req, K, V, n_out, kind, dtype, norm):
    x, xf, allowed, score, finished, eos = make(V + K, n_req, K, V, dtype, kind, norm, n_out)
    want = ref.select(xf, allowed, score, finished, eos, norm, n_req, n_out)
    check(run(wg, x, None if kind == "all" else allowed, score, finished, eos, norm, n_req, n_out), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (7, 8), (8, 24), (2, 2)])
def test_any_alignment(wg, dtype, offset, pad):
    """Rows that begin anywhere; what lies around them (NaN) is never taken for a logit."""
    for norm, kind in ((ref.NORM_ALLOWED, "most"), (ref.NORM_FULL, "few"), (ref.NORM_NONE, "all")):
        x, xf, allowed, score, finished, eos = make(5 + offset, 2, 4, 2311, dtype, kind, norm, 8)
        want = ref.select(xf, allowed, score, finished, eos, norm, 2, 8)
        check(run(wg, x, allowed, score, finished, eos, norm, 2, 8, offset, pad), want)


@pytest.mark.parametrize("n_req,K,V,n_out,dtype,kind", [
    (40, 8, 128256, 16, "bf16", "most"), (3, 4, 256000, 8, "fp32", "most"), (2, 32, 151936, 64, "bf16", "few")])
def test_large(wg, n_req, K, V, n_out, dtype, kind):
    x, xf, allowed, score, finished, eos = make(11, n_req, K, V, dtype, kind, ref.NORM_ALLOWED, n_out)
    want = ref.select(xf, allowed, score, finished, eos, ref.NORM_ALLOWED, n_req, n_out)
    check(run(wg, x, allowed, score, finished, eos, ref.NORM_ALLOWED, n_req, n_out), want)


@pytest.mark.parametrize("norm,kind", [(ref.NORM_ALLOWED, "most"), (ref.NORM_FULL, "few"), (ref.NORM_NONE, "few")])
@pytest.mark.parametrize("n_req,K,V,dtype", [
    (1, 16, 2040, "bf16"), (1, 17, 2040, "bf16"), (148, 1, 2040, "bf16"), (149, 1, 2040, "bf16"), (2, 16, 16377, "bf16"),
    (1, 8, 32761, "fp32"), (4, 16, 32760, "bf16"), (5, 16, 32760, "bf16"), (1, 17, 32760, "bf16"), (18, 4, 32761, "fp32")])
def test_one_launch_and_two(wg, n_req, K, V, dtype, norm, kind):
    """Batches on both sides of what one launch takes, at every size of its clusters."""
    x, xf, allowed, score, finished, eos = make(n_req + K, n_req, K, V, dtype, kind, norm, K)
    want = ref.select(xf, allowed, score, finished, eos, norm, n_req, K)
    check(run(wg, x, allowed, score, finished, eos, norm, n_req, K), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [ref.NORM_ALLOWED, ref.NORM_FULL, ref.NORM_NONE])
@pytest.mark.parametrize("n_out", [1, 7, 64])
def test_ties_go_to_the_lowest_index(wg, dtype, norm, n_out):
    """Every logit equal, and then two values only: far more equal scores than any list holds."""
    V, K = 20016, 3      # (rows of whole pieces: equal rows are summed in the same order)
    score = np.array([-1.0, -1.0, -1.0], np.float32)
    x = np.zeros((K, V), np.float32)
    got = run(wg, as_dtype(x, dtype), None, score, None, 0, norm, 1, n_out)
    assert got[1].tolist() == [[0] * n_out] and got[2].tolist() == [list(range(n_out))]
    rng = np.random.default_rng(3)
    x = rng.integers(0, 2, (1, V)).astype(np.float32).repeat(K, 0)       # equal rows: equal lse, bit for bit
    ones = np.flatnonzero(x[0])
    got = run(wg, as_dtype(x, dtype), None, score, None, 0, norm, 1, n_out)
    assert got[1].tolist() == [[0] * n_out] and got[2].tolist() == [ones[:n_out].tolist()]
    allowed = np.ones((K, V), bool)
    allowed[0, ones[:V // 4]] = False
    got = run(wg, as_dtype(x, dtype), allowed, score, None, 0, ref.NORM_NONE, 1, n_out)
    assert got[1].tolist() == [[0] * n_out] and got[2].tolist() == [ones[V // 4:][:n_out].tolist()]


@pytest.mark.parametrize("n_req,K,V,n_out", [(2, 4, 1000, 64), (1, 16, 1000, 32), (3, 12, 1537, 24), (1, 32, 520, 64), (1, 1, 4000, 9)])
def test_fewer_chunks_than_results(wg, n_req, K, V, n_out):
    """Nothing can be told from the chunk maxima: all elements are candidates, more than are ranked at once."""
    x, xf, allowed, score, finished, eos = make(V + K, n_req, K, V, "fp32", "most", ref.NORM_ALLOWED, n_out)
    want = ref.select(xf, allowed, score, finished, eos, ref.NORM_ALLOWED, n_req, n_out)
    check(run(wg, x, allowed, score, finished, eos, ref.NORM_ALLOWED, n_req, n_out), want)
    # with hosts of equal scores among them, on several beams, so that no bound cuts the list short
    rng = np.random.default_rng(V)
    x = as_dtype(rng.integers(-3, 2, (n_req * K, V)), "fp32")
    score = np.zeros(n_req * K, np.float32)
    want = ref.select(x.numpy(), allowed, score, np.zeros(n_req * K, bool), eos, ref.NORM_NONE, n_req, n_out)
    check(run(wg, x, allowed, score, None, eos, ref.NORM_NONE, n_req, n_out), want, 0)


def test_negative_zero_ties_with_zero(wg):
    x = np.full((1, 300), -5.0, np.float32)
    x[0, 40], x[0, 260] = -0.0, 0.0
    got = run(wg, as_dtype(x, "fp32"), None, np.zeros(1, np.float32), None, 0, ref.NORM_NONE, 1, 2)
    assert got[2].tolist() == [[40, 260]] and got[0].tolist() == [[0.0, 0.0]]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [ref.NORM_ALLOWED, ref.NORM_FULL, ref.NORM_NONE])
def test_special_values(wg, dtype, norm):
    """Infinities, NaN and the type's lowest value, allowed and masked."""
    V, K, n_out = 2500, 8, 12
    rng = np.random.default_rng(8)
    x = np.round(rng.standard_normal((K, V)) * 2048) / 1024
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    high = -low
    allowed = rng.random((K, V)) < 0.5
    masked = np.flatnonzero(~allowed[0])
    x[0, masked[:5]] = np.nan                 # NaN in a masked place
    x[1, np.flatnonzero(~allowed[1])[:3]] = np.inf
    x[2, np.flatnonzero(allowed[2])[3]] = np.nan   # NaN that counts
    x[3, np.flatnonzero(allowed[3])[3]] = np.inf
    x[4, :] = -np.inf                         # a row of nothing but -inf
    x[5, allowed[5]] = low                    # masked by the lowest value instead of -inf
    x[6, np.flatnonzero(allowed[6])[:50]] = -np.inf
    x[7, ~allowed[7]] = low
    score = np.array([-3, -2.5, -1, -4, -2, -9.25, -1.75, -6], np.float32)
    t = as_dtype(x, dtype)
    xf = t.float().numpy()
    want = ref.select(xf, allowed, score, np.zeros(K, bool), 0, norm, 1, n_out)
    got = run(wg, t, allowed, score, None, 0, norm, 1, n_out)
    check(got, want)
    # each row by itself, so that none hides behind a better one
    for b in range(K):
        want = ref.select(xf[b:b + 1], allowed[b:b + 1], score[b:b + 1], [False], 0, norm, 1, n_out)
        got = run(wg, t[b:b + 1], allowed[b:b + 1], score[b:b + 1], None, 0, norm, 1, n_out)
        if np.isfinite([s for s, _, _ in want[0]]).all() and norm != ref.NORM_NONE:
            check(got, want)
        else:
            assert got[1][0].tolist() == [p for _, p, _ in want[0]] + [-1] * (n_out - len(want[0]))
            assert got[2][0].tolist() == [p for _, _, p in want[0]] + [-1] * (n_out - len(want[0]))
    assert high > 0


def test_lowest_value_everywhere_is_uniform(wg):
    """All allowed logits at the type's lowest value: log(1 / n) each, not -inf or NaN."""
    for dtype, info in (("bf16", torch.bfloat16), ("fp32", torch.float32)):
        x = np.full((1, 700), torch.finfo(info).min, np.float64)
        got = run(wg, as_dtype(x, dtype), None, np.zeros(1, np.float32), None, 0, ref.NORM_ALLOWED, 1, 3)
        # (lse rounds to the lowest value itself: log 700 is far below its last place)
        assert got[2].tolist() == [[0, 1, 2]] and (got[0] == 0.0).all()


def test_rows_without_hypothesis_and_finished_rows(wg):
    V, K = 1500, 4
    rng = np.random.default_rng(4)
    x = as_dtype(rng.standard_normal((K, V)), "fp32")
    # the first step of a search: one beam counts
    score = np.array([0, -np.inf, -np.inf, -np.inf], np.float32)
    got = run(wg, x, None, score, None, 0, ref.NORM_ALLOWED, 1, K)
    assert (got[1] == 0).all()
    check(got, ref.select(x.numpy(), np.ones((K, V), bool), score, np.zeros(K, bool), 0, 0, 1, K))
    # all finished: their scores, in order, on EOS; logits are not looked at
    score = np.array([-3, -1, -np.inf, -2], np.float32)
    got = run(wg, torch.full((K, V), float("nan")), None, score, np.ones(K), 7, ref.NORM_FULL, 1, K)
    assert got[1].tolist() == [[1, 3, 0, -1]] and got[2].tolist() == [[7, 7, 7, -1]]
    assert got[0].tolist() == [[-1.0, -2.0, -3.0, -np.inf]]
    # NaN score: no hypothesis
    got = run(wg, x, None, np.array([np.nan, -1, np.nan, np.nan], np.float32), None, 0, ref.NORM_NONE, 1, K)
    assert (got[1] == 1).all()


def test_scores_in_place_and_reused_scratch(wg):
    """score_out over score (n_out == n_beam); a handle made for more serves smaller calls, whatever the
    call before left in it."""
    beam = wg.Beam(5000, 6, 8, 16)
    for seed, (n_req, K) in enumerate([(6, 8), (1, 2), (4, 3), (2, 8)]):
        x, xf, allowed, score, finished, eos = make(seed, n_req, K, 5000, "bf16", "few", 0, K)
        want = ref.select(xf, allowed, score, finished, eos, 0, n_req, K)
        mask = torch.from_numpy(ref.pack_mask(allowed).view(np.int32)).cuda()
        d_score = torch.from_numpy(score).cuda()
        par, tok = (torch.zeros((n_req, K), dtype=torch.int32, device="cuda") for _ in range(2))
        wg.wg_beam_select(beam, K, x.cuda(), d_score, d_score.view(n_req, K), par, tok, bitmask=mask,
                          finished=torch.from_numpy(finished.astype(np.int32)).cuda(), eos_id=eos)
        check((d_score.view(n_req, K).cpu().numpy(), par.cpu().numpy(), tok.cpu().numpy()), want)


def test_other_stream_and_graph(wg):
    """The call goes to the current stream, and can be recorded."""
    x, xf, allowed, score, finished, eos = make(2, 2, 4, 3000, "fp32", "most", 0, 4)
    want = ref.select(xf, allowed, score, finished, eos, 0, 2, 4)
    beam = wg.Beam(3000, 2, 4)
    d = dict(x=torch.zeros((8, 3000), device="cuda"), s=torch.from_numpy(score).cuda(),
             m=torch.from_numpy(ref.pack_mask(allowed).view(np.int32)).cuda(),
             f=torch.from_numpy(finished.astype(np.int32)).cuda())
    so = torch.zeros((2, 4), device="cuda")
    po, to = (torch.zeros((2, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    plan = wg.BeamPlan(beam, 4, d["s"], so, po, to, bitmask=d["m"], finished=d["f"], eos_id=eos)
    src = x.cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        d["x"].copy_(src)
        plan(d["x"])
    side.synchronize()
    check((so.cpu().numpy(), po.cpu().numpy(), to.cpu().numpy()), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan(d["x"])
    so.zero_(), po.zero_(), to.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    check((so.cpu().numpy(), po.cpu().numpy(), to.cpu().numpy()), want)


def test_refusals(wg):
    with pytest.raises(wg.WgError):
        wg.Beam(0, 1, 1)
    with pytest.raises(wg.WgError):
        wg.Beam(1000, 1, wg.WG_BEAM_MAX_BEAMS + 1)
    with pytest.raises(wg.WgError):
        wg.Beam(1000, 1, 4, wg.WG_BEAM_MAX_OUT + 1)
    with pytest.raises(wg.WgError):
        wg.Beam(1000, 65536, 1)
    beam = wg.Beam(1000, 2, 4, 8)
    x = torch.zeros((8, 1000), device="cuda")
    s = torch.zeros(8, device="cuda")
    out = lambda n=4, r=2: (torch.zeros((r, n), device="cuda"),) + tuple(  # noqa: E731
        torch.zeros((r, n), dtype=torch.int32, device="cuda") for _ in range(2))
    wg.wg_beam_select(beam, 4, x, s, *out())
    cases = [
        (ValueError, lambda: wg.wg_beam_select(beam, 3, x, s, *out())),                    # 8 rows of 3 beams
        (wg.WgError, lambda: wg.wg_beam_select(beam, 8, x, s, *out(r=1))),                 # beyond max_beams
        (wg.WgError, lambda: wg.wg_beam_select(beam, 2, x, s, *out(r=4))),                 # beyond max_requests
        (wg.WgError, lambda: wg.wg_beam_select(beam, 4, x, s, *out(9))),                   # beyond max_out
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x[:, :999], s, *out())),           # too few columns
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x[:4], s, *out())),                # too few rows
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x.t().contiguous().t(), s, *out())),
        (TypeError, lambda: wg.wg_beam_select(beam, 4, x.half(), s, *out())),
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x.cpu(), s, *out())),
        (TypeError, lambda: wg.wg_beam_select(beam, 4, x, s.double(), *out())),
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x, s, out()[0], out()[1], out(5)[2])),
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x, s, *out(), bitmask=torch.zeros((8, 31), dtype=torch.int32, device="cuda"))),
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x, s, *out(), finished=torch.zeros(8, dtype=torch.int32, device="cuda"), eos_id=1000)),
        (ValueError, lambda: wg.wg_beam_select(beam, 4, x, s, *out(), finished=torch.zeros(7, dtype=torch.int32, device="cuda"))),
        (wg.WgError, lambda: wg.wg_beam_select(beam, 4, x, s, *out(), norm=3)),
        (wg.WgError, lambda: wg.wg_beam_select(beam, 2, x[:4], s[:4], s[:4].view(2, 2)[:, :1].contiguous() * 0, *out(1)[1:], norm=-1)),
    ]
    for error, call in cases:
        with pytest.raises(error):
            call()
    b = wg.binding
    so, po, to = out()
    args = lambda **k: [dict(dict(h=beam.handle, x=x.data_ptr(), d=1, st=1000, m=None, ms=0, s=s.data_ptr(), f=None, e=0, r=2,  # noqa: E731
                                  k=4, n=4, norm=0, so=so.data_ptr(), po=po.data_ptr(), to=to.data_ptr(), stream=None), **k)[n]
                        for n in ("h", "x", "d", "st", "m", "ms", "s", "f", "e", "r", "k", "n", "norm", "so", "po", "to", "stream")]
    assert b._lib.wg_beam_select(*args()) == 0
    for bad in (dict(h=None), dict(x=None), dict(d=2), dict(st=999), dict(s=None), dict(r=0), dict(k=0), dict(n=0), dict(so=None),
                dict(po=None), dict(to=None), dict(x=x.data_ptr() + 1), dict(so=s.data_ptr(), n=8),
                dict(f=po.data_ptr(), e=-1), dict(m=po.data_ptr(), ms=31)):
        assert b._lib.wg_beam_select(*args(**bad)) == wg.WG_ERR_ARG, bad
    torch.cuda.synchronize()


@pytest.mark.parametrize("T,R,K", [(1, 1, 1), (1, 3, 4), (2, 2, 2), (7, 1, 32), (63, 5, 3), (64, 2, 8), (65, 2, 8), (513, 3, 5),
                                   (4097, 2, 8), (9000, 1, 4), (1200, 1, 32)])
def test_backtrack(wg, T, R, K):
    rng = np.random.default_rng(T * 100 + K)
    token = rng.integers(0, 1 << 20, (T, R, K)).astype(np.int32)
    parent = rng.integers(0, K, (T, R, K)).astype(np.int32)
    lost = rng.random((T, R, K)) < 0.2 / T
    parent[lost] = rng.choice([-1, K, 1 << 30], int(lost.sum()))
    out = torch.zeros((R, K, T), dtype=torch.int32, device="cuda")
    wg.wg_beam_backtrack(torch.from_numpy(token).cuda(), torch.from_numpy(parent).cuda(), out)
    assert (out.cpu().numpy() == ref.backtrack(token, parent)).all()


def test_backtrack_refusals(wg):
    t = torch.zeros((4, 2, 3), dtype=torch.int32, device="cuda")
    out = torch.zeros((2, 3, 4), dtype=torch.int32, device="cuda")
    wg.wg_beam_backtrack(t, t, out)
    wg.wg_beam_backtrack(t[:0], t[:0], out[:, :, :0].contiguous())
    for call in (lambda: wg.wg_beam_backtrack(t, t[:3], out), lambda: wg.wg_beam_backtrack(t, t, out[:, :, :3]),
                 lambda: wg.wg_beam_backtrack(t.transpose(1, 2).contiguous().transpose(1, 2), t, out),
                 lambda: wg.wg_beam_backtrack(t[0], t[0], out)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        wg.wg_beam_backtrack(t.long(), t, out)
    lib = wg.binding._lib
    p, q = t.data_ptr(), out.data_ptr()
    for bad in ((None, p, 4, 2, 3, q, None), (p, p, -1, 2, 3, q, None), (p, p, 4, 0, 3, q, None), (p, p, 4, 2, 33, q, None),
                (p, p, 4, 65536, 3, q, None)):
        assert lib.wg_beam_backtrack(*bad) == wg.WG_ERR_ARG
