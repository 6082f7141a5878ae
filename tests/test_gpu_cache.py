"""Writing into and reading out of a paged cache against plain forms."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu
BF16, FP16, E4M3, INT8, FP32 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8, torch.float32


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def bits(t):
    return t.cpu().contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def full_cache(wg, n_blocks, block, H, D, dtype, seed=0):
    """A cache with something in every place."""
    g = ref.generator(seed)
    shape = (n_blocks, block, H, D)
    planes = [torch.randint(0, 64, shape, generator=g).to(dtype).cuda() for _ in range(2)]
    if dtype in ref.LARGEST:
        planes += [torch.rand(shape[:3], generator=g).cuda() for _ in range(2)]
    return wg.KvCache(*planes)


def slot_map(wg, slot, pos):
    m = wg.SlotMap(1, len(slot))
    m.slot.copy_(torch.as_tensor(slot))
    m.pos.copy_(torch.as_tensor(pos))
    return m


def snapshot(cache):
    return [None if t is None else t.clone() for t in (cache.keys, cache.values, cache.key_scale, cache.value_scale)]


class Write:
    def __init__(self, wg, T, Hq, H, D, model, held, block=16, rot=None, interleaved=False, seed=0, most=500, **rope):
        g = ref.generator(seed + 1)
        self.rot = D if rot is None else rot
        self.T, self.Hq, self.H, self.D, self.model, self.held, self.interleaved = T, Hq, H, D, model, held, interleaved
        self.cache = full_cache(wg, T // block + 2, block, H, D, held, seed)
        n_slots = (T // block + 2) * block
        self.slot = torch.randperm(n_slots, generator=g)[:T]
        self.slot[torch.rand(T, generator=g) < 0.1] = -1
        self.pos = torch.randint(0, most, (T,), generator=g).to(torch.int32)
        new = lambda h: (torch.randn((T, h, D), generator=g) * torch.exp(torch.randn((T, h, 1), generator=g))).to(model)  # noqa: E731
        self.q, self.k, self.v = new(Hq), new(H), new(H)
        self.rope = wg.Rope(most, self.rot, interleaved=interleaved, **rope) if self.rot else None
        self.freq = self.rope.frequencies.tolist() if self.rot else []
        self.magnitude = rope.get("magnitude", 1.0)
        self.slots = slot_map(wg, self.slot, self.pos)

    def check(self, before, q_out, q_before):
        ok = self.slot >= 0
        at = self.slot[ok]
        table = None if self.rope is None else self.rope.table.cpu()
        for x, out, plane, scale, was, was_scale in (
                (self.q, q_out, None, None, q_before, None),
                (self.k, None, self.cache.keys, self.cache.key_scale, before[0], before[2]),
                (self.v, None, self.cache.values, self.cache.value_scale, before[1], before[3])):
            if x is self.q and q_out is None:
                continue
            turned = x.double() if x is self.v else ref.rotate(x, self.pos, self.freq, self.interleaved, self.magnitude)
            if plane is None:
                self.near(out.cpu()[ok], turned[ok], x[ok])
                assert torch.equal(bits(out)[~ok], bits(was)[~ok])
                continue
            got = plane.cpu().flatten(0, 1)
            rest = torch.ones(got.shape[0], dtype=torch.bool)
            rest[at] = False
            assert torch.equal(bits(got)[rest], bits(was).flatten(0, 1)[rest])
            if scale is None:
                self.near(got[at], turned[ok], x[ok])
                continue
            # 8 bits: from the same fp32 rotation the same codes and scales, to the last bit
            turned32 = x.float() if x is self.v else self.rotate32(x, table)
            codes, want_scale = ref.codes_of(turned32[ok], self.held)
            got_scale = scale.cpu().flatten(0, 1)
            assert torch.equal(bits(got_scale[at]), bits(want_scale))
            assert torch.equal(bits(got[at]), bits(codes))
            assert torch.equal(bits(got_scale)[rest], bits(was_scale).flatten(0, 1)[rest])
            # and the values held are as near as the type allows: half a step of a code, or of the smallest step
            value, top = ref.held(got[at], got_scale[at]), turned[ok].abs().amax(-1, keepdim=True)
            step = 0.5 / 127 * top if self.held is INT8 else torch.maximum(turned[ok].abs() * 2.0 ** -4, top / 448 * 2.0 ** -10)
            assert ((value - turned[ok]).abs() <= step * (1 + 2.0 ** -10) + top * 2.0 ** -22).all()

    def rotate32(self, x, table):
        if table is None:
            return x.float()
        n = self.rot // 2
        c, s = table[self.pos.long(), None, :n], table[self.pos.long(), None, n:]
        y = x.float().clone()
        a, b = (x[..., 0:self.rot:2], x[..., 1:self.rot:2]) if self.interleaved else (x[..., :n], x[..., n:2 * n])
        a, b = a.float(), b.float()
        # (a product of two fp32 numbers is exact in 64 bits)
        lo, hi = (a.double() * c - (b * s).double()).float(), (b.double() * c + (a * s).double()).float()
        if self.interleaved:
            y[..., 0:self.rot:2], y[..., 1:self.rot:2] = lo, hi
        else:
            y[..., :n], y[..., n:2 * n] = lo, hi
        return y

    def near(self, got, want, x):
        """Half a step of the result; cosine, sine and two products are off by half a step of 2^-24 each at the size of the
        pair, whose members are at most the vector's largest."""
        bound = want.abs() * ref.half_step(self.model) + x.double().abs().amax(-1, keepdim=True) * 6 * 2.0 ** -24 * max(1.0, self.magnitude)
        assert ((got.double() - want).abs() <= bound + torch.finfo(self.model).smallest_normal).all()

    def run(self, with_q=True, in_place=False):
        before = snapshot(self.cache)
        q = self.q.cuda()
        q_out = None if not with_q or in_place else torch.full_like(q, 9.0)
        was = q.clone() if in_place else None if q_out is None else q_out.clone()
        self.cache.write(self.k.cuda(), self.v.cuda(), self.slots, rope=self.rope, q=q if with_q else None, q_out=q_out)
        torch.cuda.synchronize()
        self.check(before, None if not with_q else q if in_place else q_out, was)


TYPES = [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3), (BF16, INT8), (FP16, INT8)]


@pytest.mark.parametrize("model,held", TYPES)
@pytest.mark.parametrize("Hq,H,D,rot", [(8, 2, 128, 128), (5, 5, 64, 32), (7, 1, 80, 80), (4, 1, 256, 256), (3, 3, 16, 16), (12, 4, 96, 48),
                                        (2, 1, 144, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_a_step_of_tokens(wg, model, held, Hq, H, D, rot, interleaved):
    Write(wg, 37, Hq, H, D, model, held, rot=rot, interleaved=interleaved, seed=D + Hq).run()


@pytest.mark.parametrize("model,held", TYPES)
@pytest.mark.parametrize("T", [1, 2, 700, 3001])
def test_any_number_of_tokens(wg, model, held, T):
    Write(wg, T, 8, 2, 64, model, held, seed=T).run()
    Write(wg, T, 32, 8, 64, model, held, seed=T, block=1).run(in_place=True)


@pytest.mark.parametrize("held", [BF16, E4M3])
def test_without_queries_and_without_rotation(wg, held):
    Write(wg, 50, 4, 2, 64, BF16, held).run(with_q=False)
    w = Write(wg, 50, 4, 2, 64, BF16, held, rot=0)
    w.run(with_q=False)
    w.slots.pos.fill_(-7)            # (not looked at)
    w.run(with_q=False)
    w.run()                          # (queries pass through)
    w.run(in_place=True)


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_and_scaled_frequencies(wg, interleaved):
    how = dict(base=500000.0, factor=8.0, original=8192, low=1.0, high=4.0)
    w = Write(wg, 60, 4, 2, 128, BF16, E4M3, interleaved=interleaved, most=200000, magnitude=1.25, **how)
    assert w.freq == pytest.approx(ref.frequencies(128, **how), rel=1e-14)
    w.run()
    Write(wg, 60, 4, 2, 128, FP16, FP16, interleaved=interleaved, most=200000, factor=4.0).run()


@pytest.mark.parametrize("n_pos,rot,magnitude", [(1, 16, 1.0), (1000, 64, 0.5), (300001, 128, 1.0)])
def test_tables_of_angles(wg, n_pos, rot, magnitude):
    r = wg.Rope(n_pos, rot, magnitude=magnitude)
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * torch.tensor(ref.frequencies(rot), dtype=torch.float64)
    want = torch.cat([torch.cos(angle), torch.sin(angle)], 1) * magnitude
    # one rounding to fp32, of a value whose angle (fp64) is off by its own rounding
    off = (r.table.cpu().double() - want).abs()
    assert (off <= want.abs() * 2.0 ** -24 + angle.repeat(1, 2) * 2.0 ** -51 + 2.0 ** -50).all()


@pytest.mark.parametrize("model", [BF16, FP16])
@pytest.mark.parametrize("held", [E4M3, INT8])
def test_vectors_of_any_size(wg, model, held):
    """Zeros, the smallest and largest values, one large value among small ones, infinities and NaN."""
    top = torch.finfo(model).max
    vectors = [0.0, -0.0, 1.0, top, torch.finfo(model).smallest_normal, torch.finfo(model).tiny * 2.0 ** -4, 2.0 ** -14, 1e-5]
    x = torch.tensor(vectors).to(model)[:, None, None].expand(len(vectors), 2, 32).clone()
    x[:, 1] *= torch.linspace(-1, 1, 32).to(model)
    special = torch.ones((4, 2, 32), dtype=model)
    special[0, 0, 5], special[1, 1, 31], special[2, 0, 0], special[3, 0, 7] = math.inf, math.nan, -math.inf, math.nan
    x = torch.cat([x, special])
    T = x.shape[0]
    cache = full_cache(wg, 2, 16, 2, 32, held)
    cache.write(x.cuda(), x.cuda(), slot_map(wg, range(T), [0] * T))
    codes, scale = ref.codes_of(x, held)
    for plane, s in ((cache.keys, cache.key_scale), (cache.values, cache.value_scale)):
        got, s = plane.cpu().flatten(0, 1)[:T], s.cpu().flatten(0, 1)[:T]
        assert torch.equal(torch.isnan(s), torch.isnan(scale)) and torch.equal(s[~torch.isnan(s)], scale[~torch.isnan(scale)])
        assert torch.equal(bits(got), bits(codes))
        assert torch.isnan(ref.held(got, s)[-4:]).all(2).sum(1).tolist() == [1, 1, 1, 1]      # the vector, not its neighbour
    # what stays untouched: nothing else was written
    assert (cache.keys.cpu().flatten(0, 1)[T:].float() != 0).any()


def test_infinities_and_nan_pass_through_16_bits(wg):
    x = torch.tensor([math.inf, -math.inf, math.nan, 1.0]).to(BF16).repeat(8)[None, None].contiguous()
    cache = full_cache(wg, 1, 1, 1, 32, BF16)
    cache.write(x.cuda(), x.cuda(), slot_map(wg, [0], [0]))
    assert torch.equal(torch.isnan(cache.values.cpu().view(-1)), torch.isnan(x.view(-1)))
    assert (cache.values.cpu().view(-1)[0::4] == math.inf).all() and (cache.keys.cpu().view(-1)[1::4] == -math.inf).all()


def test_slots_and_positions_out_of_range(wg):
    w = Write(wg, 12, 2, 1, 32, BF16, E4M3, most=100)
    slot = torch.tensor([0, -1, -2, 16, 31, 32, 2 ** 40, -2 ** 62, 5, 6, 7, 8])
    pos = torch.tensor([0, -1, 0, 0, 99, 0, 0, 0, -1, 100, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    assert w.cache.n_blocks * w.cache.block_size == 32
    slots = slot_map(wg, slot, pos)
    status = torch.full((12,), 5, dtype=torch.int32, device="cuda")
    before, q = snapshot(w.cache), w.q.cuda()
    w.cache.write(w.k.cuda(), w.v.cuda(), slots, rope=w.rope, q=q, status=status)
    good = [0, 3, 4]
    assert status.tolist() == [0, 0, -1, 0, 0] + [-1] * 7
    w.slot, w.pos = torch.full((12,), -1), pos.clamp(0, 99)
    w.slot[good] = slot[good]
    w.check(before, q, w.q)


def test_slots_beyond_32_bits(wg):
    """The last slots of a cache of more than 2^32 bytes and elements, and one in the middle."""
    n_blocks, block, D = (1 << 31) // 1024 + 3, 1024, 16
    cache = wg.KvCache.empty(n_blocks, block, 1, D, INT8)
    n = n_blocks * block
    x = torch.randn((3, 1, D), generator=ref.generator(1)).to(BF16)
    cache.write(x.cuda(), x.cuda(), slot_map(wg, [n - 1, 1 << 31, 7], [0] * 3))
    codes, scale = ref.codes_of(x, INT8)
    pool = wg.KvPool(n_blocks, block, 1)
    tables = wg.KvTables(pool, torch.tensor([[n_blocks - 1, (1 << 31) // block, 0]], dtype=torch.int32, device="cuda"),
                         torch.tensor([2 * block + 8], dtype=torch.int32, device="cuda"))
    out = torch.empty((2 * block + 8, 1, D), dtype=FP32, device="cuda")
    cache.read(tables, torch.tensor([0, 2 * block + 8], dtype=torch.int32, device="cuda"), out, None)
    for row, t in ((block - 1, 0), (block, 1), (2 * block + 7, 2)):
        assert torch.equal(out[row].cpu().double(), ref.held(codes, scale)[t].float().double())
    assert int((out != 0).any(2).sum()) == 3
    q = torch.zeros((1, 1, D), dtype=BF16, device="cuda")
    got = torch.empty_like(q)
    attend = wg.Attend(1, 1, 1, D)
    attend(q, cache, tables, got)    # all weights alike
    want = ref.held(codes, scale).sum(0) / (2 * block + 8)
    assert ((got[0].cpu().double() - want).abs() <= want.abs() * 2.0 ** -7 + 1e-9).all()


def test_views_of_a_fused_projection(wg):
    w = Write(wg, 40, 4, 2, 64, BF16, BF16, seed=3)
    before = snapshot(w.cache)
    fused = torch.cat([w.q.flatten(1), w.k.flatten(1), w.v.flatten(1), torch.zeros((40, 8), dtype=BF16)], 1).cuda()
    q, k, v, _ = fused.split([256, 128, 128, 8], 1)
    q, k, v = q.unflatten(1, (4, 64)), k.unflatten(1, (2, 64)), v.unflatten(1, (2, 64))
    w.cache.write(k, v, w.slots, rope=w.rope, q=q)
    w.check(before, q, w.q)
    assert torch.equal(bits(k), bits(w.k)) and torch.equal(bits(v), bits(w.v)) and (fused[:, -8:] == 0).all()


def test_no_tokens(wg):
    w = Write(wg, 40, 4, 2, 64, BF16, BF16)
    before = snapshot(w.cache)
    none = torch.empty((0, 2, 64), dtype=BF16, device="cuda")
    w.cache.write(none, none, wg.SlotMap(1, 0), rope=w.rope)
    assert torch.equal(bits(w.cache.keys), bits(before[0]))


# ---- reading back ------------------------------------------------------------------------------------------------
class Read:
    def __init__(self, wg, lens, H, D, held, block=16, seed=0):
        g = ref.generator(seed)
        self.lens, S = torch.tensor(lens, dtype=torch.int32), len(lens)
        cols = max(1, -(-max(lens) // block))
        need = sum(-(-n // block) for n in lens)
        self.cache = full_cache(wg, need + 2, block, H, D, held, seed)
        ids = torch.randperm(need + 2, generator=g).to(torch.int32)
        self.table = torch.full((S, cols), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(lens):
            c = -(-n // block)
            self.table[s, :c] = ids[at:at + c]
            at += c
        self.cu = torch.zeros(S + 1, dtype=torch.int32)
        self.cu[1:] = torch.cumsum(self.lens, 0)
        self.pool = wg.KvPool(need + 2, block, S)
        self.block = block

    def run(self, wg, dtype, spare=3, which=(True, True)):
        rows = int(self.cu[-1]) + spare
        tables = wg.KvTables(self.pool, self.table.cuda(), self.lens.cuda())
        H, D = self.cache.n_heads, self.cache.head_dim
        outs = [torch.full((rows, H, D), 7.0, dtype=dtype, device="cuda") if w else None for w in which]
        self.cache.read(tables, self.cu.cuda(), *outs)
        for out, plane, scale in zip(outs, (self.cache.keys, self.cache.values), (self.cache.key_scale, self.cache.value_scale)):
            if out is None:
                continue
            values = ref.held(plane.cpu(), None if scale is None else scale.cpu())
            want = torch.full((rows, H, D), 7.0, dtype=torch.float64)
            for s, n in enumerate(self.lens.tolist()):
                p = torch.arange(min(n, int(self.cu[s + 1] - self.cu[s])))
                entry = self.table[s].long()[(p // self.block).clamp(max=self.table.shape[1] - 1)]
                real = (entry >= 0) & (entry < self.cache.n_blocks) & (p // self.block < self.table.shape[1])
                x = values[torch.where(real, entry, 0), p % self.block]
                want[int(self.cu[s]) + p] = torch.where(real[:, None, None], x, 0.0)
            # (a product of a code and a scale is rounded to fp32 first)
            off = (out.cpu().double() - want).abs()
            assert (off <= want.abs() * (ref.half_step(dtype) + (0 if scale is None else 2.0 ** -24)) + torch.finfo(dtype).smallest_normal * 2.0 ** -8).all()


@pytest.mark.parametrize("held", [BF16, FP16, E4M3, INT8])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("H,D", [(2, 128), (1, 16), (5, 80), (8, 256)])
def test_sequences_read_back(wg, held, dtype, H, D):
    Read(wg, [0, 17, 0, 1, 16, 100, 0, 33, 0], H, D, held, seed=D).run(wg, dtype)


@pytest.mark.parametrize("block", [1, 7, 64])
@pytest.mark.parametrize("lens", [[0], [1], [0, 0, 5000], [3] * 700, list(range(200))])
def test_reads_of_any_shape(wg, block, lens):
    r = Read(wg, lens, 2, 64, E4M3, block, seed=block)
    r.run(wg, BF16)
    r.run(wg, FP32, spare=0, which=(True, False))
    r.run(wg, FP32, spare=0, which=(False, True))


def test_reads_of_broken_tables(wg):
    r = Read(wg, [40, 40, 40, 40], 2, 64, INT8)
    r.table[0, 1], r.table[1, 0], r.table[2, 2] = -1, r.cache.n_blocks, 2 ** 31 - 1
    r.run(wg, BF16)
    r.lens[3] = 100                   # beyond the table, and beyond its rows
    r.run(wg, BF16)
    r.cu[4] = int(r.cu[3]) + 100
    r.run(wg, BF16)


def test_fewer_rows_than_sequences_have(wg):
    r = Read(wg, [40, 40], 2, 64, BF16)
    out = torch.full((50, 2, 64), 7.0, dtype=BF16, device="cuda")
    tables = wg.KvTables(r.pool, r.table.cuda(), r.lens.cuda())
    r.cache.read(tables, r.cu.cuda(), out[:45], None)
    assert (out[45:] == 7).all() and (out[:45] != 7).any()


def test_recorded_and_on_another_stream(wg):
    w = Write(wg, 30, 4, 2, 64, BF16, E4M3, seed=5)
    k, v, q = w.k.cuda(), w.v.cuda(), w.q.cuda()
    q_out = torch.full_like(q, 9.0)
    before, was = snapshot(w.cache), q_out.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    w.cache.write(k, v, w.slots, rope=w.rope, q=q, q_out=q_out, stream=side)
    side.synchronize()
    w.check(before, q_out, was)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.cache.write(k, v, w.slots, rope=w.rope, q=q, q_out=q_out)
    w.slot = w.slot.roll(1)
    w.pos = w.pos.flip(0)
    w.slots.slot.copy_(w.slot)
    w.slots.pos.copy_(w.pos)
    q_out.fill_(9.0)
    before = snapshot(w.cache)
    graph.replay()
    w.check(before, q_out, was)


# ---- a step of a model's layer, as it is used ----------------------------------------------------------------------
@pytest.mark.parametrize("model,held", [(BF16, BF16), (FP16, INT8), (BF16, E4M3)])
def test_prompts_steps_beams_and_reads_together(wg, model, held):
    """Prompts of two requests written, decoded by three beams each with changing parents, cut back; after every step the
    attention of the step's tokens against a copy of what every hypothesis was given."""
    g = ref.generator(11)
    R, K, Hq, H, D, block = 2, 3, 4, 2, 64, 8
    N = R * K
    pool = wg.KvPool(120, block, N)
    table = torch.full((N, 12), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(N, dtype=torch.int32, device="cuda")
    tables = wg.KvTables(pool, table, lens, torch.zeros(N, dtype=torch.int32, device="cuda"))
    cache = full_cache(wg, 120, block, H, D, held)
    rope, attend = wg.Rope(100, 32), wg.Attend(N * 40, Hq, H, D)
    given = [[] for _ in range(N)]                      # (k, v) of every token of every hypothesis, unrotated

    def step(n_new, group):
        T = sum(n_new) + 1                              # (one place too many)
        slots = wg.SlotMap(N, T)
        tables.extend(torch.tensor(n_new, dtype=torch.int32, device="cuda"), slots)
        q, k, v = (torch.randn((T, h, D), generator=g).to(model) for h in (Hq, H, H))
        q_rot, out = q.cuda(), torch.empty((T, Hq, D), dtype=model, device="cuda")
        cache.write(k.cuda(), v.cuda(), slots, rope=rope, q=q_rot)
        attend(q_rot, cache, tables, out, slots=slots, group=group)
        t = 0
        for s in range(N):
            for _ in range(n_new[s]):
                given[s].append((k[t], v[t]))
                kk = torch.stack([x for x, _ in given[s]])
                vv = torch.stack([x for _, x in given[s]])
                pos = torch.arange(len(given[s]))
                kk = ref.rotate(kk, pos, ref.frequencies(32), False)
                if held in ref.LARGEST:
                    kk, vv = ref.held(*ref.codes_of(kk, held)), ref.held(*ref.codes_of(vv, held))
                else:
                    kk = kk.to(held)
                qq = ref.rotate(q[t][None], pos[-1:], ref.frequencies(32), False).to(model)
                one = torch.arange(len(given[s]), dtype=torch.int32)[None]
                want, _, mass, size = ref.attend(qq, kk.double()[:, None], vv.double()[:, None], one, [0], [len(given[s]) - 1], D ** -0.5)
                tol, _ = ref.tolerance(want, mass, size, [len(given[s])], D, model, held if held in (BF16, FP16) else FP16,
                                       None if held not in ref.LARGEST else torch.ones(1))
                # rotated keys may round the other way: one step of what is held, in a score, and so twice in a weight
                steps = {BF16: 2.0 ** -7, FP16: 2.0 ** -10, E4M3: 2.0 ** -3, INT8: 2.0 ** -6}[held]
                flips = size[0] * steps / 8
                assert ((out[t].cpu().double() - want[0]).abs() <= tol[0] + 2 * flips[:, None] * mass[0]).all()
                t += 1
        assert (out[T - 1] == 0).all()
        return out

    step([21, 0, 0, 30, 0, 0], 1)
    parents = torch.tensor([[0, 0, 0], [0, 0, 0]], dtype=torch.int32, device="cuda")
    for i in range(12):
        tables.reorder(parents, cache.planes)
        flat = (torch.arange(R)[:, None] * K + parents.cpu()).view(-1).tolist()
        given[:] = [list(given[p]) for p in flat]
        step([1] * N, K)
        parents = torch.randint(0, K, (R, K), generator=g).to(torch.int32).cuda()
    # (the last token lies in a block of the sequence's own: what is shared must not be written to)
    step([1] * N, 1)
    tables.shrink(torch.tensor([len(x) - 1 for x in given], dtype=torch.int32, device="cuda"))
    given[:] = [x[:-1] for x in given]
    step([2] * N, 2)
    cu = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    cu[1:] = torch.cumsum(lens, 0)
    assert lens.tolist() == [len(x) for x in given]
    v_out = torch.empty((int(cu[-1]), H, D), dtype=FP32, device="cuda")
    cache.read(tables, cu, None, v_out)
    want = torch.cat([torch.stack([v for _, v in x]) for x in given])
    want = ref.held(*ref.codes_of(want, held)) if held in ref.LARGEST else want.double()
    assert ((v_out.cpu().double() - want).abs() <= want.abs() * 2.0 ** -23).all()
