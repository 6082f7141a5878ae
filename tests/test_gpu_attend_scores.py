"""Attention over a paged cache with scores far beyond what a softmax usually sees.

Queries and keys have one dimension that is not 0 and holds few bits, so that every dot product is exact in fp32.  Scores
then differ by 0 or by so much that a row's result is the mean of the values at its largest score: a case of few roundings."""
import math
import sys

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu
BF16, FP16, E4M3, INT8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8
TYPES = [(BF16, BF16), (FP16, FP16), (E4M3, BF16), (E4M3, FP16), (INT8, BF16), (INT8, FP16)]
D, ROWS = 64, 16


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


class Far:
    """Sequences of one key head.  Row r of a token has the query 2^12 (1 + r / 16) in one dimension, with a sign; the key
    at a position is one of `n_keys` steps of a type's largest ones there (key 0 the largest)."""

    def __init__(self, wg, lens, held, model, size, sign, n_keys, rows=ROWS, seed=0, share=False):
        g = ref.generator(seed)
        self.lens, self.rows, self.model, self.held, narrow = lens, rows, model, held, held in ref.LARGEST
        n_blocks = sum(-(-n // 16) for n in lens)
        shape = (n_blocks, 16, 1, D)
        steps = {E4M3: torch.tensor([448.0, 416, 384, 352, 320, 288, 256, 240, 224, 208]), INT8: 127.0 - torch.arange(32)}.get(
            held, 2.0 ** 12 * (1 - torch.arange(32) / 64))
        which = torch.randint(0, n_keys, shape[:3], generator=g)
        k = torch.zeros(shape)
        k[..., 0] = steps[which]
        if narrow:
            self.ks = torch.full(shape[:3], 2.0 ** 4)
            self.vs = torch.exp2(torch.randint(-6, 7, shape[:3], generator=g).float())
            self.v = torch.randint(1, 120, shape, generator=g).float().to(held)
        else:
            self.ks = self.vs = None
            self.v = torch.randn(shape, generator=g).to(held)
        self.k = k.to(held)
        self.q = torch.zeros((len(lens), rows, D))
        self.q[..., 0] = sign * 2.0 ** 12 * (1 + torch.arange(rows) / 16)
        self.q = self.q.to(model)
        largest = float(ref.held(self.k, self.ks).max()) * 2.0 ** 12
        self.scale = 2.0 ** round(math.log2(size / largest))
        ids = torch.randperm(n_blocks, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), -(-max(lens) // 16)), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(lens):
            self.table[s, :-(-n // 16)] = ids[at:at - (-n // 16)]
            at += -(-n // 16)
        if share:                        # of the longest
            at = lens.index(max(lens))
            self.table = torch.where(self.table < 0, -1, self.table[at])
        put = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.cache = wg.KvCache(*(put(t) for t in (self.k, self.v, self.ks, self.vs)))
        self.pool = wg.KvPool(n_blocks, 16, len(lens))
        self.tables = wg.KvTables(self.pool, self.table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        self.attend = wg.Attend(len(lens), rows, 1, D)

    def run(self, group=1):
        out = torch.full(self.q.shape, 7.0, dtype=self.model, device="cuda")
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        self.attend(self.q.cuda(), self.cache, self.tables, out, scale=self.scale, lse=lse, group=group)
        return out.cpu().double(), lse.cpu().double()

    def check(self, group=1):
        out, lse = self.run(group)
        keys, values = ref.held(self.k, self.ks), ref.held(self.v, self.vs)
        for s, n in enumerate(self.lens):
            p = torch.arange(n)
            k, v = keys[self.table[s].long()[p // 16], p % 16, 0], values[self.table[s].long()[p // 16], p % 16, 0]
            for r in range(self.rows):
                x = (k @ self.q[s, r].double()) * self.scale
                first = x == x.max()
                assert first.all() or x.max() - x[~first].max() > 100
                want, mass = v[first].mean(0), v[first].abs().mean(0)
                # Weights are 2^(log2 of a scale less that of another) at most: the logarithms of powers of two and the exponential are
                # off by 2^-21 each, an exponent of up to 32 by its last step, 2^-19; sums by a step of 2^-24 each; fp16 weights by half
                # a step (16-bit ones are exact: 1).
                rel = 3 * 2.0 ** -19 + int(first.sum()) * 2.0 ** -23 + (ref.half_step(FP16) if self.held in ref.LARGEST else 0)
                off = (out[s, r] - want).abs()
                assert (off <= want.abs() * ref.half_step(self.model) + mass * rel).all(), (s, r, (off / mass).max().item())
                # scale, log2(e), their product, two products with it, a sum and the way back to natural logarithms, a step each
                want = x.max().item() + math.log(int(first.sum()))
                assert abs(lse[s, r].item() - want) <= abs(want) * 8 * 2.0 ** -24 + 2.0 ** -16


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("size", [1e5, 1.2e7, 1e8, 3e10, 1e12])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores(wg, held, model, size, sign):
    """Few positions, some thousand that are split between blocks and joined, alone and in groups."""
    s = Far(wg, [1, 40, 700, 3000], held, model, size, sign, 8)
    for group in (1, 2, 4):
        s.check(group)
    Far(wg, [1, 40, 700, 3000], held, model, size, sign, 8, share=True).check(4)


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("size", [1.2e7, 5e7, 1e12])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores_that_are_all_alike(wg, held, model, size, sign):
    """All keys of a sequence are one: every position counts the same, whatever the size of its value."""
    s = Far(wg, [3, 40, 3000, 200], held, model, size, sign, 1, seed=1)
    for group in (1, 4):
        s.check(group)
    Far(wg, [3, 40, 3000, 200], held, model, size, sign, 1, seed=1, share=True).check(4)


@pytest.mark.parametrize("held,model", [(BF16, BF16), (FP16, FP16), (E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("rows", [4, 40])
def test_large_scores_by_other_kernels(wg, held, model, rows):
    """Few rows and many, and so many sequences that warps work by themselves."""
    s = Far(wg, [50] * 3 + [2000], held, model, 1.2e7, 1, 8, rows, seed=2)
    s.check()
    s.check(4)
    s = Far(wg, [1 + i % 40 for i in range(700)], held, model, 5e7, 1, 4, min(rows, 16), seed=3)
    s.lens = s.lens[:30]             # (the others are only there to be many)
    s.check()


def scores(wg, held, rows):
    """Rows of a 16-bit cache of one head: [(query, keys)] of one dimension, scale 4; results of position p's value p + 1."""
    n = max(len(k) for _, k in rows)
    keys, values = torch.zeros((len(rows), n, 1, D)), torch.zeros((len(rows), n, 1, D))
    q = torch.zeros((len(rows), 1, D))
    for s, (x, k) in enumerate(rows):
        q[s, 0, 0] = x
        keys[s, :len(k), 0, 0] = torch.tensor(k)
        values[s, :, 0] = torch.arange(1.0, n + 1)[:, None]
    cache = wg.KvCache(keys.to(held).cuda(), values.to(held).cuda())
    pool = wg.KvPool(len(rows), n, len(rows))
    tables = wg.KvTables(pool, torch.arange(len(rows), dtype=torch.int32, device="cuda")[:, None].contiguous(),
                         torch.tensor([len(k) for _, k in rows], dtype=torch.int32, device="cuda"))
    out, lse = torch.empty((len(rows), 1, D), dtype=held, device="cuda"), torch.empty((len(rows), 1), device="cuda")
    wg.Attend(len(rows), 1, 1, D)(q.to(held).cuda(), cache, tables, out, scale=4.0, lse=lse)
    return out.cpu()[:, 0], lse.cpu()[:, 0]


@pytest.mark.parametrize("n", [3, 400])
def test_scores_beyond_fp32(wg, n):
    """A score that is +inf in fp32 makes its row NaN; -inf has no weight, and where all are, nothing is left: whether a row was split or not."""
    out, lse = scores(wg, BF16, [(2.0 ** 63, [2.0 ** 64] + [1.0] * n), (2.0 ** 63, [-2.0 ** 64] * n), (2.0 ** 63, [-2.0 ** 64] * n + [0.0]),
                                 (2.0 ** 100, [2.0 ** 100] * n), (2.0 ** 100, [-2.0 ** 100] * n), (1.0, [0.0] * n)])
    assert torch.isnan(out[[0, 3]]).all() and torch.isnan(lse[[0, 3]]).all()
    assert (out[[1, 4]] == 0).all() and (lse[[1, 4]] == -math.inf).all()
    assert (out[2] == torch.tensor(n + 1.0).to(BF16)).all() and lse[2] == 0
    assert torch.isfinite(out[5]).all() and abs(lse[5].item() - math.log(n)) < 1e-5


@pytest.mark.parametrize("held,size,scale", [(BF16, 2.0 ** 60, 0.0), (BF16, 2.0 ** 60, 1e-39), (BF16, 2.0 ** 60, -2e-38), (E4M3, 2.0 ** 60, 0.0), (INT8, 2.0 ** 60, 1e-38),
                                             (INT8, 2.0 ** 60, -2e-38), (FP16, 2.0 ** 14, 0.0)])
def test_scales_of_nothing(wg, held, size, scale):
    """Dot products near the end of fp32's range times a scale of 0, or next to it."""
    model = FP16 if held is FP16 else BF16
    g = ref.generator(9)
    q, k = torch.zeros((3, 4, D)), torch.zeros((3, 64, 1, D))
    q[..., 0] = size * (1 + torch.arange(4) / 4)
    k[..., 0] = size * torch.randn((3, 64, 1), generator=g)
    v = torch.randn((3, 64, 1, D), generator=g)
    if held in ref.LARGEST:
        (k, ks), (v, vs) = ref.codes_of(k, held), ref.codes_of(v, held)
    else:
        k, v, ks, vs = k.to(held), v.to(held), None, None
    put = lambda t: None if t is None else t.cuda()  # noqa: E731
    cache, pool = wg.KvCache(*(put(t) for t in (k, v, ks, vs))), wg.KvPool(3, 64, 3)
    tables = wg.KvTables(pool, torch.arange(3, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.full((3,), 60, dtype=torch.int32, device="cuda"))
    out, lse = torch.empty((3, 4, D), dtype=model, device="cuda"), torch.empty((3, 4), device="cuda")
    wg.Attend(3, 4, 1, D)(q.to(model).cuda(), cache, tables, out, scale=scale, lse=lse)
    x = torch.einsum("srd,spd->srp", q.to(model).double(), ref.held(k, ks)[:, :60, 0]) * scale
    values, w = ref.held(v, vs)[:, :60, 0], torch.softmax(x, 2)
    mean, mass = w @ values, w @ values.abs()
    # half a step of a weight and of the result; scores of some units, whose factors have at least 2^17 steps below fp32's normal range
    assert ((out.cpu().double() - mean).abs() <= mean.abs() * ref.half_step(model) + mass * (ref.half_step(BF16 if held is BF16 else FP16) + 2.0 ** -14)).all()
    assert ((lse.cpu().double() - torch.logsumexp(x, 2)).abs() <= 2.0 ** -14).all()


@pytest.mark.parametrize("held", [E4M3, INT8])
def test_keys_of_zeros_beside_the_largest_queries(wg, held):
    """A query's size and the scale together are beyond fp32; its scores are 0."""
    v = torch.randn((1, 16, 1, D), generator=ref.generator(10))
    (k, ks), (v, vs) = ref.codes_of(torch.zeros((1, 16, 1, D)), held), ref.codes_of(v, held)
    cache, pool = wg.KvCache(*(t.cuda() for t in (k, v, ks, vs))), wg.KvPool(1, 16, 1)
    tables = wg.KvTables(pool, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.full((1,), 16, dtype=torch.int32, device="cuda"))
    out, lse = torch.empty((1, 4, D), dtype=BF16, device="cuda"), torch.empty((1, 4), device="cuda")
    wg.Attend(1, 4, 1, D)(torch.full((1, 4, D), 2.0 ** 127, device="cuda").to(BF16), cache, tables, out, scale=64.0, lse=lse)
    mean = ref.held(v, vs)[0, :, 0].mean(0)
    mass = ref.held(v, vs)[0, :, 0].abs().mean(0)
    assert ((out.cpu().double() - mean).abs() <= mean.abs() * 2.0 ** -8 + mass * (2.0 ** -11 + 2.0 ** -18)).all()
    assert (lse.cpu().double() - math.log(16)).abs().max() < 1e-5


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("dim", [80, 128, 256])
@pytest.mark.parametrize("rows", [4, 12, 20])
def test_large_scores_at_other_head_sizes(wg, held, model, dim, rows, monkeypatch):
    monkeypatch.setattr(sys.modules[__name__], "D", dim)
    for share, n_keys in ((False, 8), (True, 8), (False, 1)):
        s = Far(wg, [1, 40, 300, 1200], held, model, 1.2e7, 1, n_keys, rows, seed=dim, share=share)
        s.check()
        s.check(4)


@pytest.mark.parametrize("held,model", [(BF16, BF16), (FP16, FP16), (E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("window", [1, 16, 50])
@pytest.mark.parametrize("new", [2, 5])
def test_drafted_tokens_under_a_window(wg, held, model, window, new):
    from test_gpu_attend import Setup
    s = Setup(wg, [1, 0, 2, 17, 64, 130, 300], 8, 2, 64, held, model, seed=new, new=new).on_gpu()
    for group in (1, new):
        s.check(s.run(window=window, group=group), window)
