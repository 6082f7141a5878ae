"""Attention over 8-bit caches whose values have scales of any size, none, or no number."""
import math

import pytest
import torch

import cache_ref as ref
from test_gpu_attend import Setup

pytestmark = pytest.mark.gpu
BF16, FP16, E4M3, INT8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def same_tables(lens):
    """All sequences on the first columns of the longest."""
    longest = lens.index(max(lens))
    return {i: (longest, -(-n // 16)) for i, n in enumerate(lens) if i != longest}


def check_lse(s, lse, window=0, scale=None):
    """The scores' sum has no values in it: as with values of 1."""
    scale = s.scale if scale is None else scale
    ones = torch.ones(s.v.shape, dtype=torch.float64)
    want, want_lse, mass, size = ref.attend(s.q, ref.held(s.k, s.ks), ones, s.table, s.seq, s.pos, scale, window)
    # (scales enter by their logarithms, no larger than 128)
    _, tol = ref.tolerance(want, mass, size, (s.pos + 1).clamp(min=1), s.D, s.model, FP16, torch.tensor([2.0 ** -128]))
    empty = want_lse == -math.inf
    assert (lse[empty] == -math.inf).all()
    off = (lse.double() - want_lse)[~empty].abs()
    assert (off <= tol.expand_as(want_lse)[~empty]).all(), off.max().item()


def far_below(s):
    """Scores of about -240, all alike."""
    s.q.zero_()
    s.q[..., 0] = -400.0
    s.k.zero_()
    s.k[..., 0] = torch.tensor(96.0).to(s.held)
    s.ks.fill_(0.05)
    s.scale = 0.125


@pytest.mark.parametrize("held,model", [(E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("window", [0, 1])
@pytest.mark.parametrize("lens", [[1, 40, 0, 300, 2500], [1 + i % 70 for i in range(80)]])
def test_values_without_a_number(wg, held, model, low, window, lens):
    """No visible value has one: every result is NaN, and the scores' sum is what it is."""
    for share in (None, same_tables(lens)):
        s = Setup(wg, lens, 8, 2, 64, held, model, seed=1, share=share)
        if low:
            far_below(s)
        s.vs.fill_(math.nan)
        s.on_gpu()
        for group in (1, 5):
            out, lse = s.run(window=window, group=group, scale=s.scale)
            some = s.lens > 0
            assert torch.isnan(out[some]).all() and (out[~some] == 0).all()
            check_lse(s, lse, window)


@pytest.mark.parametrize("held,model", [(E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("lens", [[1, 40, 0, 300, 2500], [1 + i % 70 for i in range(80)]])
def test_a_value_without_a_number(wg, held, model, bad, lens):
    """One of each sequence's, of the first head: NaN everywhere, or infinite where its code is not 0."""
    for share in (None, same_tables(lens)):
        s = Setup(wg, lens, 8, 2, 64, held, model, seed=2, share=share)
        clean = Setup(wg, lens, 8, 2, 64, held, model, seed=2, share=share).on_gpu()
        at = {}
        for i, n in enumerate(lens):
            if n:
                p = (0 if share else 3 * n // 4)
                at[i] = (int(s.table[i, p // 16]), p % 16)
                s.vs[at[i]][0] = bad
        s.on_gpu()
        for group in (1, 5):
            (out, lse), (want, _) = s.run(group=group), clean.run(group=group)
            check_lse(s, lse)
            for i, (b, o) in at.items():
                code = s.v[b, o, 0].float()
                first = torch.where(code == 0, math.nan, torch.sign(code) * bad).expand(4, -1)
                assert torch.equal(torch.isnan(out[i, :4]), torch.isnan(first))
                assert torch.equal(out[i, :4].float()[~torch.isnan(first)], first[~torch.isnan(first)])
                assert torch.equal(out[i, 4:], want[i, 4:])


@pytest.mark.parametrize("held", [E4M3, INT8])
def test_values_of_infinite_scale_alone(wg, held):
    """Tokens that see one position, and tokens that see nothing else."""
    lens = [1, 1, 30, 2000]
    s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=3)
    s.vs.fill_(math.inf)
    s.v.fill_(2.0) if held is E4M3 else s.v.fill_(2)
    s.v[..., 1::2] = torch.tensor(-3.0).to(held)
    s.on_gpu()
    for group in (1, 2):
        out, lse = s.run(group=group)
        assert (out[..., 0::2] == math.inf).all() and (out[..., 1::2] == -math.inf).all()
        check_lse(s, lse)


@pytest.mark.parametrize("held", [E4M3, INT8])
@pytest.mark.parametrize("size", [-70, -85, -98])
def test_values_as_small_as_are_written(wg, held, size):
    """Vectors of about 2^size, written by the library: codes and scales as for any other."""
    lens = [1, 40, 0, 700, 3000]
    s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=4)
    slots = wg.SlotMap(1, s.n_blocks * 16)
    slots.slot.copy_(torch.arange(s.n_blocks * 16))
    g = ref.generator(size + 1000)
    k, v = (torch.randn((s.n_blocks * 16, 2, 64), generator=g) for _ in range(2))
    v = v * torch.exp2(size + 4 * torch.rand((s.n_blocks * 16, 2, 1), generator=g))
    s.on_gpu()
    s.cache.write(k.to(BF16).cuda(), v.to(BF16).cuda(), slots)
    (s.k, s.ks), (s.v, s.vs) = (ref.codes_of(x.to(BF16).view(s.n_blocks, 16, 2, 64), held) for x in (k, v))
    assert torch.equal(s.cache.value_scale.cpu(), s.vs) and (s.vs < 2.0 ** (size + 2)).all()
    for group in (1, 5):
        s.check(s.run(group=group))


def lost(s):
    """What fp16 weights may lose beside the largest.  A weight is exp(x[i] - lse) times the value's scale, divided by the largest of
    the row and times 2^15.  Below 2^-14 it is off by up to half of fp16's smallest step, 2^-25, which is 2^-40 of the largest,
    whatever it is itself, and that times the code in the result.  (It is seen in dimensions where the largest's code is 0.)"""
    out = torch.zeros(s.q.shape, dtype=torch.float64)
    keys = ref.held(s.k, s.ks)
    G = s.Hq // s.H
    for t in range(s.q.shape[0]):
        p = torch.arange(int(s.pos[t]) + 1)
        b = s.table[int(s.seq[t])].long()[p // 16]
        for h in range(s.Hq if len(p) else 0):
            weight = torch.softmax(keys[b, p % 16, h // G] @ s.q[t, h].double() * s.scale, 0) * s.vs[b, p % 16, h // G].double()
            out[t, h] = 2.0 ** -40 * weight.max() * s.v[b, p % 16, h // G].double().abs().sum(0)
    return out


@pytest.mark.parametrize("held", [E4M3, INT8])
@pytest.mark.parametrize("low,high", [(-100, -95), (-120, -110), (-110, 0), (-120, 110)])
def test_value_scales_over_the_whole_range(wg, held, low, high):
    for lens in ([1, 40, 0, 700, 3000], [1 + i % 70 for i in range(80)]):
        s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=5)
        s.vs = torch.exp2(torch.randint(low, high + 1, s.vs.shape, generator=ref.generator(high)).float()) * s.vs.clamp(0.5, 2.0)
        s.on_gpu()
        want, want_lse, mass, size = s.want()
        tol, tol_lse = ref.tolerance(want, mass, size, (s.pos + 1).clamp(min=1), 64, BF16, FP16, s.vs)
        tol += lost(s)
        for group in (1, 5):
            out, lse = s.run(group=group)
            off, some = (out.double() - want).abs(), s.lens > 0
            assert (off <= tol).all(), ((off / tol).max().item(), int((off > tol).sum()))
            assert ((lse.double() - want_lse)[some].abs() <= tol_lse[some]).all() and (lse[~some] == -math.inf).all()


@pytest.mark.parametrize("held,largest", [(E4M3, 448.0), (INT8, 127.0)])
def test_values_as_large_as_there_are(wg, held, largest):
    """One vector of bf16's largest values among ordinary ones."""
    lens = [1, 40, 0, 700, 3000]
    s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=6)
    for i, n in enumerate(lens):
        if n:
            p = 2 * n // 3
            b = int(s.table[i, p // 16])
            top = torch.full((2, 64), torch.finfo(BF16).max) * torch.sign(torch.randn((2, 64), generator=ref.generator(i)))
            s.v[b, p % 16], s.vs[b, p % 16] = ref.codes_of(top.to(BF16), held)
    s.on_gpu()
    want, want_lse, mass, size = s.want()
    tol, tol_lse = ref.tolerance(want, mass, size, (s.pos + 1).clamp(min=1), 64, BF16, FP16, s.vs)
    # beside a scale of 2^k the sum has no weights below 2^(k - 138) of the largest
    keys, left_out = ref.held(s.k, s.ks), torch.zeros(5, 8, dtype=torch.float64)
    for t, n in enumerate(lens):
        p = torch.arange(n)
        b = s.table[t].long()[p // 16]
        for h in range(8 if n else 0):
            w = torch.softmax(keys[b, p % 16, h // 4] @ s.q[t, h].double() * s.scale, 0)
            left_out[t, h] = w[w < w.max() * 2.0 ** (math.log2(torch.finfo(BF16).max / largest) - 138)].sum()
    assert left_out.max() < 2.0 ** -8
    tol, tol_lse = tol + lost(s) + 2 * left_out[..., None] * mass, tol_lse + 2 * left_out
    for group in (1, 5):
        out, lse = s.run(group=group)
        assert ((out.double() - want).abs() <= tol).all()
        assert ((lse.double() - want_lse)[s.lens > 0].abs() <= tol_lse[s.lens > 0]).all()


@pytest.mark.parametrize("held", [E4M3, INT8])
@pytest.mark.parametrize("size", [1e-6, 1e-9, 2.0 ** -60])
@pytest.mark.parametrize("lens", [[2, 40, 0, 700, 3000], [2 + i % 70 for i in range(80)]])
def test_a_vector_of_zeros_has_no_part(wg, held, size, lens):
    """Zeros are written with the scale 1.  One that nearly all of the weight lies on leaves the small ones beside it their bits; so do
    minus zeros; and vectors whose scale happens to be 1 count as they are."""
    for share in (None, same_tables(lens)):
        s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=7, share=share)
        g = ref.generator(7)
        slots = wg.SlotMap(1, s.n_blocks * 16)
        slots.slot.copy_(torch.arange(s.n_blocks * 16))
        k = torch.randn((s.n_blocks, 16, 2, 64), generator=g)
        v = size * (1 + torch.rand((s.n_blocks, 16, 2, 64), generator=g)) * torch.sign(torch.randn((s.n_blocks, 16, 2, 64), generator=g))
        for i, n in enumerate(lens):
            for p in {n // 2, n - 1} if n else ():
                k[s.table[i, p // 16], p % 16] = s.q[i].float().view(2, 4, 64).mean(1) * 3
                v[s.table[i, p // 16], p % 16] = 0.0 if p == n - 1 else -0.0
        s.on_gpu()
        k, v = k.to(BF16), v.to(BF16)
        s.cache.write(k.cuda().flatten(0, 1), v.cuda().flatten(0, 1), slots)
        (s.k, s.ks), (s.v, s.vs) = ref.codes_of(k, held), ref.codes_of(v, held)
        assert (s.vs == 1).any() and s.vs.min() < size
        for group in (1, 5):
            s.check(s.run(group=group))


@pytest.mark.parametrize("held", [E4M3, INT8])
def test_scales_of_one(wg, held):
    for lens in ([1, 40, 0, 700, 3000], [1 + i % 70 for i in range(80)]):
        s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=8)
        s.vs.fill_(1.0)
        s.on_gpu()
        for group in (1, 5):
            s.check(s.run(group=group))


def any_scales(s, seed):
    """Scales of values from 2^-100 to 2^60, some 1, some of those with zeros; keys a hundred times as large in one sequence."""
    g = ref.generator(seed)
    s.vs = torch.exp2(torch.randint(-100, 61, s.vs.shape, generator=g).float()) * s.vs.clamp(0.5, 2.0)
    s.vs[torch.rand(s.vs.shape, generator=g) < 0.3] = 1.0
    s.v.view(torch.uint8)[(s.vs == 1) & (torch.rand(s.vs.shape, generator=g) < 0.5)] = 0
    for c in range(s.table.shape[1]):
        if s.table[3, c] >= 0:
            s.ks[s.table[3, c]] *= 100.0


@pytest.mark.parametrize("held,model", [(E4M3, BF16), (INT8, BF16)])
@pytest.mark.parametrize("D", [80, 128, 256])
@pytest.mark.parametrize("rows", [4, 12, 20])
def test_unusual_tiles_at_other_head_sizes(wg, held, model, D, rows):
    """Single tokens of few and of many sequences, drafted tokens, and beams that share a block."""
    some = [1, 40, 0, 500, 90]
    for lens, new, share in ((some, 1, None), ([1 + i % 70 for i in range(40)] * 2, 1, None), (some, 3, None), (some, 1, same_tables(some))):
        s = Setup(wg, lens, 2 * rows, 2, D, held, model, seed=D, new=new, share=share)
        any_scales(s, D + rows)
        s.on_gpu()
        few = torch.arange(0, s.q.shape[0], 1 if len(lens) == 5 else 11)
        got = {group: s.run(group=group) for group in ((1,) if len(lens) > 5 else (1, 5, new))}
        s.q, s.seq, s.pos = s.q[few], s.seq[few], s.pos[few]
        want, want_lse, mass, size = s.want()
        tol, tol_lse = ref.tolerance(want, mass, size, (s.pos + 1).clamp(min=1), D, model, FP16, s.vs)
        tol = tol + lost(s)
        seen = s.pos >= 0
        for out, lse in got.values():
            off = (out[few].double() - want).abs()
            assert (off <= tol).all(), ((off / tol).max().item(), int((off > tol).sum()))
            assert ((lse[few].double() - want_lse)[seen].abs() <= tol_lse[seen]).all() and (lse[few][~seen] == -math.inf).all()


@pytest.mark.parametrize("held,model", [(E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_without_a_number_at_other_head_sizes(wg, held, model, D, bad):
    """Beams that share a block and end at different places before, at and behind one without a number."""
    lens = [70, 75, 79, 72, 0, 40]
    s = Setup(wg, lens, 8, 2, D, held, model, seed=33, share=same_tables(lens))
    clean = Setup(wg, lens, 8, 2, D, held, model, seed=33, share=same_tables(lens)).on_gpu()
    s.vs[int(s.table[2, 4]), 73 - 64] = bad
    s.on_gpu()
    for group in (1, 2, 6):
        (out, lse), (want, want_lse) = s.run(group=group), clean.run(group=group)
        assert torch.equal(out[[0, 3, 4, 5]], want[[0, 3, 4, 5]]) and torch.equal(lse[[0, 3, 4, 5]], want_lse[[0, 3, 4, 5]])
        assert not torch.isfinite(out[[1, 2]]).any()
        check_lse(s, lse)


@pytest.mark.parametrize("held", [E4M3, INT8])
@pytest.mark.parametrize("exponent", [None, -93, -99])
@pytest.mark.parametrize("n", [1 << 17, (1 << 21) + 5, 1 << 27])
def test_very_many_values_of_next_to_nothing(wg, held, exponent, n):
    """Zeros (None) or vectors of about 2^exponent at every position, the same block over and over: the scores' sum counts them all."""
    block, H, D, cols = 1 << 16, 1, 16, -(-n // (1 << 16))
    g = ref.generator(12)
    v = torch.zeros((block, H, D)) if exponent is None else torch.randn((block, H, D), generator=g) * 2.0 ** exponent
    k = torch.zeros((block, H, D))
    cache = wg.KvCache(*(torch.zeros((1, block, H, D), dtype=held, device="cuda") for _ in range(2)),
                       *(torch.ones((1, block, H), device="cuda") for _ in range(2)))
    slots = wg.SlotMap(1, block)
    slots.slot.copy_(torch.arange(block))
    cache.write(k.to(BF16).cuda(), v.to(BF16).cuda(), slots)
    pool = wg.KvPool(1, block, 3)
    lens = [n, 1000, 0]
    tables = wg.KvTables(pool, torch.zeros((3, cols), dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = torch.randn((3, 4, D), generator=g).to(BF16).cuda()
    held_v = ref.held(*ref.codes_of(v.to(BF16), held))[:, 0]
    attend = wg.Attend(3, 4, H, D)
    for group in (1, 3):
        out, lse = torch.full_like(q, 7.0), torch.full((3, 4), 7.0, device="cuda")
        attend(q, cache, tables, out, lse=lse, group=group)
        for s, m in enumerate(lens):
            want = (held_v.sum(0) * (m // block) + held_v[:m % block].sum(0)) / max(m, 1)
            mass = (held_v.abs().sum(0) * (m // block) + held_v[:m % block].abs().sum(0)) / max(m, 1)
            # weights of 2^3 and less in fp16 of fp32 sums of some hundred thousand terms each
            rel = ref.half_step(FP16) + 2.0 ** 18 * 2.0 ** -23 * (m > 1000) + 2.0 ** -13
            assert ((out[s].cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 + mass * rel + 2.0 ** -133).all()
            assert ((lse[s].cpu().double() - (math.log(m) if m else -math.inf)).abs() <= 2.0 ** 18 * 2.0 ** -23).all() if m else (lse[s] == -math.inf).all()
