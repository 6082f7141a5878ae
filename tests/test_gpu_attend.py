"""Attention over a paged cache against a plain 64-bit form."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu
BF16, FP16, E4M3, INT8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


class Setup:
    """Sequences of the given lengths on blocks in no order, a full cache, and one token per sequence (or more)."""

    def __init__(self, wg, lens, Hq, H, D, held=BF16, model=BF16, block=16, seed=0, spare=2, share=None, new=1):
        g = ref.generator(seed)
        self.wg, self.held, self.model, self.block, self.Hq, self.H, self.D = wg, held, model, block, Hq, H, D
        S = len(lens)
        self.lens = torch.tensor(lens, dtype=torch.int32)
        cols = max(1, -(-max(lens) // block)) + 1
        need = sum(-(-n // block) for n in lens)
        self.n_blocks = need + spare
        ids = torch.randperm(self.n_blocks, generator=g).to(torch.int32)
        self.table = torch.full((S, cols), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(lens):
            c = -(-n // block)
            self.table[s, :c] = ids[at:at + c]
            at += c
        for s, (of, columns) in (share or {}).items():       # sequence s has the first columns of another
            self.table[s, :columns] = self.table[of, :columns]
        shape = (self.n_blocks, block, H, D)
        strong = torch.exp(0.5 * torch.randn(shape[2:], generator=g))
        k = torch.randn(shape, generator=g) * strong
        v = torch.randn(shape, generator=g) * torch.exp(torch.randn(shape[:3], generator=g))[..., None]
        if held in ref.LARGEST:
            (self.k, self.ks), (self.v, self.vs) = ref.codes_of(k, held), ref.codes_of(v, held)
        else:
            self.k, self.v, self.ks, self.vs = k.to(held), v.to(held), None, None
        T = S * new
        self.seq = torch.arange(T, dtype=torch.int32) // new
        self.pos = self.lens[self.seq.long()] - new + torch.arange(T, dtype=torch.int32) % new
        self.pos[self.pos < 0] = -1
        self.q = (torch.randn((T, Hq, D), generator=g) * 1.5).to(model)
        self.scale, self.new = D ** -0.5, new

    def on_gpu(self):
        wg, put = self.wg, lambda t: None if t is None else t.cuda()  # noqa: E731
        self.cache = wg.KvCache(put(self.k), put(self.v), put(self.ks), put(self.vs))
        self.pool = wg.KvPool(self.n_blocks, self.block, len(self.lens))
        self.tables = wg.KvTables(self.pool, put(self.table), put(self.lens))
        self.attend = wg.Attend(self.q.shape[0], self.Hq, self.H, self.D)
        self.slots = wg.SlotMap(len(self.lens), self.q.shape[0])
        self.slots.seq.copy_(self.seq)
        self.slots.pos.copy_(self.pos)
        self.slots.slot.copy_(torch.where(self.pos < 0, -1, 0))
        return self

    def run(self, mapped=False, q=None, out=None, **how):
        T = self.q.shape[0]
        q = self.q.cuda() if q is None else q
        out = torch.full((T, self.Hq, self.D), 7.0, dtype=self.model, device="cuda") if out is None else out
        lse = torch.full((T, self.Hq), 7.0, device="cuda")
        self.attend(q, self.cache, self.tables, out, slots=self.slots if mapped or self.new > 1 else None, lse=lse, **how)
        torch.cuda.synchronize()
        return out.cpu(), lse.cpu()

    def want(self, window=0, scale=None):
        scale = self.scale if scale is None else scale
        return ref.attend(self.q, ref.held(self.k, self.ks), ref.held(self.v, self.vs), self.table, self.seq, self.pos, scale, window)

    def check(self, got, window=0, scale=None):
        out, lse = got
        want, want_lse, mass, size = self.want(window, scale)
        weights = self.held if self.held in (BF16, FP16) else FP16
        tol, tol_lse = ref.tolerance(want, mass, size, (self.pos + 1).clamp(min=1), self.D, self.model, weights, self.vs)
        off = (out.double() - want).abs()
        assert torch.isfinite(out.double()).all()
        assert (off <= tol).all(), f"{(off / tol).max().item():.2f} of the bound, {(off > tol).sum().item()} values"
        empty = want_lse == -math.inf
        assert (lse[empty] == -math.inf).all() and (out[empty] == 0).all()
        off = (lse.double() - want_lse)[~empty].abs()
        assert (off <= tol_lse.expand_as(want_lse)[~empty]).all(), f"lse off by {off.max().item():.3g}"
        return (off.max().item() if off.numel() else 0.0)


LENS = [1, 0, 2, 15, 16, 17, 63, 64, 65, 130, 300, 0, 513]


@pytest.mark.parametrize("held,model", [(BF16, BF16), (FP16, FP16), (E4M3, BF16), (E4M3, FP16), (INT8, BF16), (INT8, FP16)])
@pytest.mark.parametrize("Hq,H,D", [(8, 2, 128), (5, 5, 64), (7, 1, 80), (4, 1, 256), (2, 1, 16), (12, 4, 96), (6, 3, 144)])
def test_one_token_each(wg, held, model, Hq, H, D):
    s = Setup(wg, LENS, Hq, H, D, held, model, seed=Hq * D).on_gpu()
    s.check(s.run())


@pytest.mark.parametrize("block", [1, 7, 8, 16, 64, 100])
@pytest.mark.parametrize("held", [BF16, E4M3])
def test_blocks_of_any_size(wg, held, block):
    s = Setup(wg, LENS, 8, 2, 128, held, block=block, seed=block).on_gpu()
    s.check(s.run())


@pytest.mark.parametrize("rows", [1, 3, 8, 15, 16, 17, 24, 33, 64, 71])
@pytest.mark.parametrize("held", [FP16, INT8])
def test_any_number_of_heads_of_a_key(wg, held, rows):
    s = Setup(wg, [40, 0, 700, 5], 2 * rows, 2, 64, held, FP16, seed=rows).on_gpu()
    s.check(s.run())


@pytest.mark.parametrize("held,model", [(BF16, BF16), (E4M3, FP16), (INT8, BF16)])
@pytest.mark.parametrize("window", [1, 2, 16, 17, 100, 513, 1000])
def test_windows(wg, held, model, window):
    s = Setup(wg, LENS, 8, 2, 64, held, model, seed=window).on_gpu()
    s.check(s.run(window=window), window)
    s.check(s.run(window=window, group=4), window)
    s = Setup(wg, [700, 20], 40, 1, 64, held, model, seed=window).on_gpu()
    s.check(s.run(window=window), window)


@pytest.mark.parametrize("n", [4000, 9001])
@pytest.mark.parametrize("held", [BF16, FP16, E4M3, INT8])
def test_long_rows_are_split_and_joined(wg, held, n):
    model = held if held in (BF16, FP16) else BF16
    s = Setup(wg, [n], 4, 2, 128, held, model, seed=n).on_gpu()
    first = s.run()
    s.check(first)
    for _ in range(3):               # whichever block comes last
        again = s.run()
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("group", [2, 4, 13])
def test_groups_of_sequences_without_anything_in_common(wg, held, group):
    s = Setup(wg, LENS, 8, 2, 128, held, seed=group).on_gpu()
    s.check(s.run(group=group))
    s.check(s.run(mapped=True, group=group))


@pytest.mark.parametrize("held,model", [(BF16, BF16), (FP16, FP16), (E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("Hq,H,D", [(8, 2, 128), (4, 4, 64), (40, 2, 64), (6, 1, 80), (8, 1, 256)])
@pytest.mark.parametrize("beams", [2, 5, 12])
def test_beams_with_a_prompt_in_common(wg, held, model, Hq, H, D, beams):
    """Three requests; the beams of each share columns, whole or none; lengths differ, some beams have ended."""
    lens, share = [], {}
    for r, (prompt, columns) in enumerate([(200, 10), (33, 2), (16, 0)]):
        for b in range(beams):
            lens.append(0 if (r * beams + b) % 7 == 3 else prompt + (b * 5) % 23)
            if b and columns:
                share[r * beams + b] = (r * beams, columns)
    if lens[0] == 0 or lens[beams] == 0:
        lens[0], lens[beams] = 200, 33
    share = {s: x for s, x in share.items() if lens[s] > 0}
    s = Setup(wg, lens, Hq, H, D, held, model, seed=beams, share=share).on_gpu()
    s.check(s.run(group=beams))


@pytest.mark.parametrize("beams,prompt", [(8, 5000), (3, 3000), (32, 700)])
@pytest.mark.parametrize("held", [BF16, E4M3])
def test_long_prompts_in_common(wg, held, beams, prompt):
    share = {b: (0, prompt // 16) for b in range(1, beams)}
    s = Setup(wg, [prompt + 7 * b for b in range(beams)], 8, 2, 64, held, seed=beams, share=share).on_gpu()
    first = s.run(group=beams)
    s.check(first)
    again = s.run(group=beams)
    assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
    s.check(s.run())


@pytest.mark.parametrize("dead", [(0,), (3,), (1, 2, 6), (0, 7)])
def test_ended_beams_beside_long_ones(wg, dead):
    """Beams that have ended, or have only just begun, beside others whose prompt many blocks work on."""
    lens = [0 if b in dead else 6000 + b for b in range(8)]
    lens[4] = 20
    first = next(b for b in range(8) if lens[b])
    s = Setup(wg, lens, 8, 2, 64, seed=21, share={b: (first, lens[b] // 16 if b == 4 else 370) for b in range(8) if lens[b] and b != first}).on_gpu()
    s.check(s.run(group=8))
    s.check(s.run(group=4))


@pytest.mark.parametrize("held", [BF16, FP16, INT8])
@pytest.mark.parametrize("new", [2, 5])
@pytest.mark.parametrize("group", [1, 0])
def test_drafted_tokens(wg, held, new, group):
    """A drafted token does not see those behind it, whatever they hold."""
    model = held if held in (BF16, FP16) else BF16
    s = Setup(wg, LENS + [900], 8, 2, 128, held, model, seed=new, new=new).on_gpu()
    s.check(s.run(group=group or new))


def test_a_group_at_the_end_that_is_not_full(wg):
    s = Setup(wg, [50, 60, 70, 80, 90], 8, 2, 64, seed=3, share={1: (0, 3), 4: (3, 4)}).on_gpu()
    for group in (2, 3, 4, 32):
        s.check(s.run(group=group))


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2100])
@pytest.mark.parametrize("group", [1, 2])
def test_more_tokens_than_a_launch_takes(wg, n, group):
    g = ref.generator(n)
    lens = torch.randint(0, 20, (n,), generator=g).tolist()
    s = Setup(wg, lens, 2, 1, 16, seed=n).on_gpu()
    s.check(s.run(group=group))
    s.check(s.run(mapped=True, group=group))


@pytest.mark.parametrize("held", [BF16, E4M3])
def test_what_is_not_seen_has_no_effect(wg, held):
    """NaN and infinities behind the last position, before the window, in other blocks and in the sequences that share blocks."""
    lens = [37, 100, 64, 0, 101]
    s = Setup(wg, lens, 8, 2, 64, held, seed=5, share={4: (1, 6)})
    clean = Setup(wg, lens, 8, 2, 64, held, seed=5, share={4: (1, 6)}).on_gpu()
    seen = torch.zeros((s.n_blocks, 16), dtype=torch.bool)
    for i, n in enumerate(lens):
        for p in range(max(0, n - 50), n):
            seen[s.table[i, p // 16], p % 16] = True
    bad = torch.tensor([math.nan, math.inf, -math.inf])[torch.arange(s.n_blocks * 16) % 3].view(s.n_blocks, 16)
    if held is E4M3:
        for t in (s.ks, s.vs):
            t[~seen] = bad[~seen][:, None]
        for t in (s.k, s.v):
            t.view(torch.uint8)[~seen] = 0x7F
    else:
        for t in (s.k, s.v):
            t[~seen] = bad[~seen][:, None, None].to(held)
    s.on_gpu()
    for group in (1, 5):
        got, want = s.run(window=50, group=group), clean.run(window=50, group=group)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("held", [BF16, INT8])
def test_a_drafted_token_does_not_see_the_next_ones_nan(wg, held):
    s = Setup(wg, [70, 33], 8, 2, 64, held, seed=9, new=3)
    for i, n in enumerate([70, 33]):
        b, o = int(s.table[i, (n - 1) // 16]), (n - 1) % 16
        if held is INT8:
            s.vs[b, o], s.ks[b, o] = math.nan, math.nan
        else:
            s.v[b, o], s.k[b, o] = math.nan, math.nan
    s.on_gpu()
    for group in (1, 3):
        out, lse = s.run(group=group)
        for t in range(6):
            last = t % 3 == 2
            assert torch.isnan(out[t]).all() == last and torch.isnan(out[t]).any() == last
            assert torch.isnan(lse[t]).all() == last and torch.isnan(lse[t]).any() == last


@pytest.mark.parametrize("group", [1, 4])
def test_nan_and_infinite_scores_stay_in_their_row(wg, group):
    s = Setup(wg, [300, 300, 300, 300], 8, 2, 64, BF16, seed=2, share={1: (0, 18), 2: (0, 18), 3: (0, 18)})
    s.q[1, 3] = math.nan
    s.q[2, 0] = math.inf
    s.on_gpu()
    out, lse = s.run(group=group)
    for t in range(4):
        for h in range(8):
            bad = (t, h) in ((1, 3), (2, 0))
            assert torch.isnan(out[t, h]).all() == bad and torch.isnan(lse[t, h]) == bad


def test_scores_of_minus_infinity(wg):
    """All of a row's scores -inf: nothing is left; some of them: they have no weight."""
    s = Setup(wg, [40, 40], 2, 1, 64, BF16, seed=4)
    s.q.fill_(1.0)
    s.k.fill_(1.0)
    for p in range(40):
        s.k[s.table[0, p // 16], p % 16] = -math.inf
        if p % 3:
            s.k[s.table[1, p // 16], p % 16] = -math.inf
    s.on_gpu()
    out, lse = s.run()
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    keep = [p for p in range(40) if p % 3 == 0]
    want = torch.stack([s.v[s.table[1, p // 16], p % 16, 0].double() for p in keep]).mean(0)
    mass = torch.stack([s.v[s.table[1, p // 16], p % 16, 0].double().abs() for p in keep]).mean(0)
    assert ((out[1].double() - want).abs() <= want.abs() * 2.0 ** -8 + mass * (2.0 ** -8 + 2.0 ** -18)).all()
    assert (lse[1].double() - (8.0 + math.log(len(keep)))).abs().max() < 1e-4


@pytest.mark.parametrize("held", [BF16, E4M3])
def test_entries_that_are_no_block(wg, held):
    """Inside a sequence: passed over, whatever they are, for one row and for a group."""
    s = Setup(wg, [100, 100, 40, 17], 8, 2, 64, held, seed=6, share={1: (0, 7)})
    s.table[0, 2] = s.table[1, 2] = -1
    s.table[0, 4], s.table[1, 5] = s.n_blocks, 2 ** 31 - 1
    s.table[2, :] = -5
    s.table[3, 0] = -2 ** 31
    s.on_gpu()
    s.check(s.run())
    s.check(s.run(group=2))
    s.check(s.run(group=4))


def test_tokens_without_a_row(wg):
    s = Setup(wg, [50, 60, 70, 80], 4, 2, 64, seed=8)
    s.seq = torch.tensor([-1, 4, 1, 2, 3, 0, 2 ** 31 - 1, 2], dtype=torch.int32)
    s.pos = torch.tensor([3, 3, -1, 10 ** 6, 2 ** 31 - 1, 49, 0, 5], dtype=torch.int32)
    s.q = torch.randn((8, 4, 64), generator=ref.generator(1)).to(BF16)
    s.on_gpu()
    s.slots.slot.copy_(torch.tensor([0, 0, 0, 0, 0, 1, 0, 2]))
    s.check(s.run(mapped=True))
    s.check(s.run(mapped=True, group=3))
    s.slots.slot[7] = -1             # refused: it has no row either
    out, lse = s.run(mapped=True)
    assert (out[7] == 0).all() and (lse[7] == -math.inf).all() and (out[5] != 0).any()


def test_lengths_beyond_the_table(wg):
    s = Setup(wg, [50, 60], 4, 2, 64, seed=8)
    s.on_gpu()
    s.tables.lens.copy_(torch.tensor([s.table.shape[1] * 16 + 1, 60]))
    s.pos[0] = -1
    s.check(s.run())
    s.check(s.run(group=2))


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("held", [FP16, E4M3])
def test_scales(wg, held, scale):
    s = Setup(wg, [50, 300], 4, 2, 64, held, FP16, seed=8).on_gpu()
    s.check(s.run(scale=scale), scale=scale)


@pytest.mark.parametrize("held", [E4M3, INT8])
def test_value_scales_of_any_size(wg, held):
    """The weight lies on positions whose values are small beside those of others, or have no scale at all."""
    s = Setup(wg, [200, 90], 4, 2, 64, held, BF16, seed=11)
    s.vs *= torch.exp2(torch.randint(-60, 40, s.vs.shape, generator=ref.generator(3)).float())
    s.vs[s.vs < 2.0 ** -40] = 0.0
    s.on_gpu()
    out, lse = s.run()
    want, want_lse, mass, size = s.want()
    tol, tol_lse = ref.tolerance(want, mass, size, s.pos + 1, 64, BF16, FP16, s.vs.clamp(min=2.0 ** -80))
    assert ((out.double() - want).abs() <= tol).all()
    assert ((lse.double() - want_lse).abs() <= tol_lse + 100 * 2.0 ** -22).all()
    for t in range(2):               # nearly all of the weight on one position with small values
        q, p = s.q[t, 0].float(), 5
        b, o = int(s.table[t, 0]), p
        s.k[b, o, 0] = torch.sign(q).to(torch.float32).mul(100).to(s.k.dtype)
        s.ks[b, o, 0], s.vs[b, o, 0] = 0.02, 2.0 ** -50
    s.on_gpu()
    out, lse = s.run()
    want, want_lse, mass, size = s.want()
    tol, _ = ref.tolerance(want, mass, size, s.pos + 1, 64, BF16, FP16, s.vs.clamp(min=2.0 ** -80))
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e4, 1e30])
def test_queries_of_any_size(wg, size):
    s = Setup(wg, [90, 30], 4, 2, 64, INT8, BF16, seed=12)
    s.q = (s.q.double() * size).to(BF16)
    s.on_gpu()
    s.check(s.run(scale=0.125 / size), scale=0.125 / size)


def test_rows_any_distance_apart_and_in_place(wg):
    s = Setup(wg, [50, 0, 300, 64], 8, 2, 64, seed=13).on_gpu()
    want = s.run()
    fused = torch.full((4, 3 * 8 * 64 + 8), 3.0, dtype=BF16, device="cuda")
    q = fused[:, 8:8 + 512].unflatten(1, (8, 64))
    q.copy_(s.q)
    out = fused[:, 520 + 8:520 + 8 + 512].unflatten(1, (8, 64))
    got = s.run(q=q, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    rest = torch.ones_like(fused, dtype=torch.bool)
    rest[:, 8:520] = False
    rest[:, 528:1040] = False
    assert (fused[rest] == 3.0).all()
    got = s.run(q=q, out=q)          # into the queries
    assert torch.equal(got[0], want[0])
    long = Setup(wg, [9000], 8, 2, 64, seed=14).on_gpu()
    want, q = long.run(), long.q.cuda()
    assert torch.equal(long.run(q=q, out=q)[0], want[0])


def test_rows_behind_the_last_are_left_alone(wg):
    s = Setup(wg, [50, 40], 4, 2, 64, seed=15).on_gpu()
    out = torch.full((3, 4, 64), 5.0, dtype=BF16, device="cuda")
    lse = torch.full((3, 4), 5.0, device="cuda")
    s.attend(s.q.cuda(), s.cache, s.tables, out[:2], lse=lse[:2])
    assert (out[2] == 5).all() and (lse[2] == 5).all() and (out[:2] != 5).all()
    s.attend(s.q[:1].cuda(), s.cache, s.tables, out[2:])       # fewer tokens than sequences
    assert torch.equal(out[2], out[0])


def test_other_streams_and_recorded_calls(wg):
    s = Setup(wg, [500, 40, 0, 3000], 8, 2, 128, seed=16).on_gpu()
    want = s.run()
    side = torch.cuda.Stream()
    q, out = s.q.cuda(), torch.zeros((4, 8, 128), dtype=BF16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.attend(q, s.cache, s.tables, out)
    side.synchronize()
    assert torch.equal(out.cpu(), want[0])
    out.zero_()
    torch.cuda.synchronize()
    s.attend(q, s.cache, s.tables, out, stream=side)
    side.synchronize()
    assert torch.equal(out.cpu(), want[0])
    for group in (1, 4):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(3):
                s.attend(q, s.cache, s.tables, out, group=group)
        for lens in ([500, 40, 0, 3000], [1, 700, 33, 2900], [0, 0, 0, 0]):
            s.tables.lens.copy_(torch.tensor(lens))
            graph.replay()
            got = out.cpu()
            assert torch.equal(got, s.run(group=group)[0])
        s.tables.lens.copy_(s.lens)


def test_calls_one_after_the_other_share_the_scratch(wg):
    a = Setup(wg, [5000, 40, 800, 3000], 8, 2, 128, seed=17).on_gpu()
    b = Setup(wg, [70, 4000, 1, 600], 8, 2, 128, seed=18, share={1: (0, 4)}).on_gpu()
    b.attend = a.attend
    want = [a.run(), b.run(group=2)]
    outs = [torch.empty((4, 8, 128), dtype=BF16, device="cuda") for _ in range(20)]
    qa, qb = a.q.cuda(), b.q.cuda()
    for i, out in enumerate(outs):
        s, q, group = ((a, qa, 1), (b, qb, 2))[i % 2]
        a.attend(q, s.cache, s.tables, out, group=group)
    for i, out in enumerate(outs):
        assert torch.equal(out.cpu(), want[i % 2][0])


def test_codes_that_are_nan_and_the_smallest(wg):
    """e4m3's NaN in a key or a value of one position; int8's -128, which this library does not write."""
    s = Setup(wg, [40, 40], 4, 2, 64, E4M3, seed=30)
    b = int(s.table[0, 1])
    s.k.view(torch.uint8)[b, 3, 0, 5] = 0x7F
    s.v.view(torch.uint8)[b, 4, 1, 7] = 0xFF
    s.on_gpu()
    out, lse = s.run()
    assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all()               # the key's head
    assert torch.isnan(out[0, 2:, 7]).all() and int(torch.isnan(out[0, 2:]).sum()) == 2 and torch.isfinite(lse[0, 2:]).all()
    assert torch.isfinite(out[1]).all()
    s = Setup(wg, [40, 40], 4, 2, 64, INT8, seed=31)
    s.k[int(s.table[0, 0]), 2], s.v[int(s.table[1, 2]), 1] = -128, -128
    s.on_gpu()
    s.check(s.run())


@pytest.mark.parametrize("held", [BF16, FP16, E4M3, INT8])
def test_the_end_of_a_shared_tile_holds_nan_for_some(wg, held):
    """Beams that share a block and end at different places in it; what lies behind the shorter ones' ends is NaN or infinite for
    the longer ones, and nothing to the shorter."""
    model = held if held in (BF16, FP16) else BF16
    lens = [70, 75, 79, 72]
    s = Setup(wg, lens, 8, 2, 64, held, model, seed=32, share={b: (2, 5) for b in (0, 1, 3)})
    clean = Setup(wg, lens, 8, 2, 64, held, model, seed=32, share={b: (2, 5) for b in (0, 1, 3)}).on_gpu()
    b = int(s.table[2, 4])
    if held in (E4M3, INT8):
        s.vs[b, 73 - 64], s.vs[b, 76 - 64] = math.nan, math.inf
    else:
        s.v[b, 73 - 64], s.v[b, 76 - 64] = math.nan, math.inf
    s.on_gpu()
    for group in (2, 4):
        out, want = s.run(group=group)[0], clean.run(group=group)[0]
        assert torch.equal(out[[0, 3]], want[[0, 3]])                  # 70 and 72 positions
        assert not torch.isfinite(out[1]).any() and not torch.isfinite(out[2]).any()
    clean.check(clean.run(group=4))
