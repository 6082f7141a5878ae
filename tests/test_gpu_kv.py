"""Block tables of a paged cache against plain lists (all results are whole numbers or moved bytes: exact)."""
import numpy as np
import pytest
import torch

import beam_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


class Both:
    """The same calls on the library and on the plain tables, compared after each."""

    def __init__(self, wg, n_blocks, block, n_seq, max_blocks, stride=None):
        self.wg, self.plain = wg, ref.Tables(n_blocks, block, n_seq, max_blocks)
        self.pool = wg.KvPool(n_blocks, block, n_seq)
        self.store = torch.full((n_seq, stride or max_blocks), -1, dtype=torch.int32, device="cuda")
        self.lens, self.status = i32(np.zeros(n_seq)), i32(np.full(n_seq, 99))
        self.tables = wg.KvTables(self.pool, self.store[:, :max_blocks], self.lens, self.status)
        self.n_seq = n_seq

    def same(self):
        torch.cuda.synchronize()
        assert (self.tables.table.cpu().numpy() == self.plain.table()).all()
        assert self.lens.tolist() == self.plain.len
        assert self.pool.ref.tolist() == self.plain.ref
        assert self.pool.n_free() == len(self.plain.free())

    def extend(self, new, n_tokens):
        m = self.wg.SlotMap(self.n_seq, n_tokens)
        self.tables.extend(i32(new), m)
        want = self.plain.extend([int(n) for n in new], n_tokens)
        for got, w, what in zip((m.cu, m.slot, m.pos, m.seq, self.status), want, ("cu", "slot", "pos", "seq", "status")):
            assert (got.cpu().numpy() == w).all(), what
        self.same()
        return m

    def shrink(self, keep):
        st = i32(np.full(self.n_seq, 99))
        self.tables.shrink(i32(keep), status=st)
        assert (st.cpu().numpy() == self.plain.shrink([int(k) for k in keep])).all()
        self.same()

    def reorder(self, parent, planes=None):
        src, dst = i32(np.full(self.n_seq, 99)), i32(np.full(self.n_seq, 99))
        before = None if planes is None else [p.clone() for p in planes]
        self.tables.reorder(i32(parent), None if planes is None else self.wg.KvPlanes(planes, self.plain.block), src, dst)
        copies, w_src, w_dst, w_st = self.plain.reorder(np.asarray(parent))
        assert (src.cpu().numpy() == w_src).all() and (dst.cpu().numpy() == w_dst).all()
        assert (self.status.cpu().numpy() == w_st).all()
        if planes is not None:
            for p, b in zip(planes, before):
                for s, d, n in copies:
                    b[d, :n] = b[s, :n]
                assert torch.equal(p, b)
        self.same()


@pytest.mark.parametrize("block", [1, 3, 16, 64])
@pytest.mark.parametrize("n_seq", [1, 5, 70, 1500])
def test_random_life(wg, n_seq, block):
    """Rounds of growing and cutting, with the pool running out now and then."""
    rng = np.random.default_rng(n_seq * 7 + block)
    max_blocks = 20
    both = Both(wg, max(3, n_seq * 6), block, n_seq, max_blocks, stride=max_blocks + 3)
    for step in range(8):
        new = rng.integers(0, 4 * block + 2, n_seq)
        new[rng.random(n_seq) < 0.3] = 0
        if step % 3 == 2:
            new[rng.random(n_seq) < 0.1] = rng.choice([-1, 20 * block + 1, 2 ** 31 - 1])
        room = int(np.clip(new, 0, 4 * block + 2).sum())
        both.extend(new, room + 5 if step % 2 else max(1, room * 3 // 4))
        keep = (np.array(both.plain.len) * rng.random(n_seq)).astype(np.int64)
        same = rng.random(n_seq) < 0.6
        keep[same] = np.array(both.plain.len)[same]
        if step % 3 == 1:
            keep[rng.random(n_seq) < 0.1] = rng.choice([-1, 1 << 20])
        both.shrink(keep)


@pytest.mark.parametrize("n_tokens", [0, 1, 2047, 2048, 2049, 9000])
def test_slots_of_few_and_many_tokens(wg, n_tokens):
    both = Both(wg, 4000, 4, 3, 3000)
    third = n_tokens // 3
    both.extend([third, 0, n_tokens - third], n_tokens)
    both.extend([1, 1, 1], 3)


def test_many_blocks(wg):
    """More blocks than one round of the search for free ones covers (262 144), nearly all held."""
    n = 700_001
    pool = wg.KvPool(n, 16, 4)
    ref_counts = torch.ones(n, dtype=torch.int32, device="cuda")
    free = [3, 262143, 262144, 262145, 524287, 524288, 699999, 700000]
    ref_counts[free] = 0
    pool.load(ref_counts)
    assert pool.n_free() == len(free)
    table, lens = i32(np.full((4, 8), -1)), i32(np.zeros(4))
    st = i32(np.zeros(4))
    t = wg.KvTables(pool, table, lens, st)
    m = wg.SlotMap(4, 16 * 9)
    t.extend(i32([33, 16, 0, 65]), m)
    assert st.tolist() == [0, 0, 0, -3] and table[0, :4].tolist() == free[:3] + [-1] and table[1, :2].tolist() == [262145, -1]
    assert m.slot[:49].tolist() == [b * 16 + i for b in free[:4] for i in range(16)][:33] + [262145 * 16 + i for i in range(16)]
    t.extend(i32([0, 0, 64, 0]), m)
    assert table[2].tolist() == free[4:] + [-1] * 4 and pool.n_free() == 0
    assert int(m.slot[63]) == 700000 * 16 + 15
    t.shrink(i32([0, 0, 0, 0]))
    assert pool.n_free() == len(free) and (table == -1).all() and torch.equal(pool.ref, ref_counts)


def test_slots_beyond_32_bits(wg):
    """Slots are 64-bit: a block number times a large block size passes 2^32."""
    bs = 1 << 20
    pool = wg.KvPool(8192, bs, 1)
    held = torch.ones(8192, dtype=torch.int32, device="cuda")
    held[8191] = 0
    pool.load(held)
    t = wg.KvTables(pool, i32([[-1]]), i32([0]))
    m = wg.SlotMap(1, 3)
    t.extend(i32([3]), m)
    assert m.slot.tolist() == [8191 * bs + i for i in range(3)]


@pytest.mark.parametrize("R,K", [(1, 1), (1, 2), (3, 4), (5, 8), (2, 32), (40, 5)])
@pytest.mark.parametrize("block", [1, 4, 16])
def test_random_search(wg, R, K, block):
    """A search's life: a prompt in one beam, a fork, then steps of one token and a selection each."""
    rng = np.random.default_rng(R * 100 + K + block)
    n = R * K
    both = Both(wg, n * 14 + 4, block, n, 300 // block + 4)
    planes = [torch.randn((n * 14 + 4, block, 24), device="cuda"), torch.randint(0, 99, (n * 14 + 4, block, 3), device="cuda", dtype=torch.uint8),
              torch.randn((n * 14 + 4, block, 2, 40), device="cuda").to(torch.bfloat16)]
    prompt = np.zeros((R, K), np.int64)
    prompt[:, 0] = rng.integers(0, 6 * block, R)
    both.extend(prompt.reshape(-1), int(prompt.sum()) + 1)
    both.reorder(np.zeros((R, K), np.int64), planes)
    for step in range(12):
        new = (rng.random(n) < 0.85).astype(np.int64)      # finished beams get no token
        both.extend(new, n)
        parent = rng.integers(0, K, (R, K))
        if step % 4 == 3:
            parent[rng.random((R, K)) < 0.15] = rng.choice([-1, K, 2 ** 31 - 1])
        both.reorder(parent, planes)
    both.shrink(np.zeros(n))
    assert both.pool.n_free() == both.plain.n_blocks


def test_no_block_left_for_a_copy(wg):
    """Four children of one parent and two free blocks: the last child is cut to its full blocks."""
    both = Both(wg, 5, 4, 4, 4)
    both.extend([6, 4, 0, 0], 10)            # two blocks and one: two free
    both.reorder([[0, 0, 0, 0]])             # beam 1's block comes free: three copies fit
    both.shrink([6, 4, 4, 4])
    both.extend([0, 4, 0, 0], 4)
    both.reorder([[0, 0, 1, 0]])
    assert both.status.tolist().count(-3) == 0
    both.extend([4, 0, 2, 0], 6)
    both.reorder([[2, 2, 2, 2]])
    both.reorder([[0, 0, 0, 0]])


def test_capacity_of_copies(wg):
    both = Both(wg, 3, 4, 4, 4)
    both.extend([6, 0, 0, 0], 6)
    both.reorder([[0, 0, 0, 0]])
    assert both.status.tolist() == [0, 0, -3, -3] and both.lens.tolist() == [6, 6, 4, 4]


def test_prefix_shared_between_requests(wg):
    """Rows of two requests that name the same blocks: counts drop once per row, free at the last."""
    pool = wg.KvPool(10, 2, 4)
    table = i32([[7, 3, -1], [7, 5, -1], [7, 2, -1], [7, -1, -1]])
    lens = i32([4, 4, 4, 2])
    counts = np.zeros(10, np.int32)
    for b in (7, 7, 7, 7, 3, 5, 2):
        counts[b] += 1
    pool.load(i32(counts))
    t = wg.KvTables(pool, table, lens, i32(np.zeros(4)))
    t.reorder(i32([[1, 1], [-1, 0]]))
    assert table.tolist() == [[7, 5, -1], [7, 5, -1], [-1, -1, -1], [7, 2, -1]] and lens.tolist() == [4, 4, 0, 4]
    assert pool.ref.tolist() == [0, 0, 1, 0, 0, 2, 0, 3, 0, 0] and pool.n_free() == 7
    t.reorder(i32([[-1, -1], [0, -1]]))
    assert pool.n_free() == 10 and pool.ref.tolist() == [0] * 10


def test_many_columns(wg):
    """Tables wider than one block of columns; a long prompt shared by all beams."""
    both = Both(wg, 3000, 2, 6, 900)
    both.extend([1501, 0, 0, 777, 0, 0], 2278)
    both.reorder([[0, 0, 0], [0, 0, 0]])
    both.extend([1] * 6, 6)
    both.reorder([[2, 1, 2], [-1, 1, 0]])


def test_planes_of_odd_sizes_and_long_rows(wg):
    both = Both(wg, 40, 8, 4, 6)
    odd = torch.randint(0, 255, (40, 8, 5), dtype=torch.uint8, device="cuda")        # 5 bytes per token
    wide = torch.randn((40, 8, 4096), device="cuda")
    both.extend([13, 0, 0, 0], 13)
    both.reorder([[0, 0, 0, 0]], [odd, wide])
    both.extend([1, 2, 3, 4], 10)
    both.reorder([[3, 2, 3, 2]], [wide, odd])


def test_counts_outlive_their_pool(wg):
    """A view of the counts keeps the memory it shows."""
    import gc
    pool = wg.KvPool(1000, 4, 2)
    pool.load(i32(np.arange(1000)))
    view = pool.ref
    owner = pool._owner
    del pool
    gc.collect()
    assert owner.value and view.tolist() == list(range(1000))
    import weakref
    gone = weakref.ref(owner)
    del owner
    assert gone() is not None
    del view
    gc.collect()
    assert gone() is None


def test_refusals(wg):
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 65536), (-5, 1, 1)):
        with pytest.raises(wg.WgError):
            wg.KvPool(*bad)
    pool = wg.KvPool(16, 4, 4)
    table, lens = i32(np.full((4, 5), -1)), i32(np.zeros(4))
    t = wg.KvTables(pool, table, lens)
    m = wg.SlotMap(4, 8)
    cases = [
        (ValueError, lambda: wg.KvTables(pool, i32(np.zeros((5, 2))), i32(np.zeros(5)))),    # more than max_seqs
        (TypeError, lambda: wg.KvTables(pool, table.long(), lens)),
        (ValueError, lambda: wg.KvTables(pool, table, lens[:3])),
        (ValueError, lambda: wg.KvTables(pool, table.t(), lens)),
        (ValueError, lambda: t.extend(i32([1, 1, 1]), m)),
        (ValueError, lambda: t.extend(torch.zeros(4, dtype=torch.int64, device="cuda"), m)),
        (ValueError, lambda: t.extend(torch.zeros(4, dtype=torch.int32), m)),
        (ValueError, lambda: t.extend(i32([1, 1, 1, 1]), wg.SlotMap(3, 8))),
        (ValueError, lambda: t.shrink(i32([0, 0]))),
        (ValueError, lambda: t.reorder(i32([0, 0, 0, 0]))),
        (ValueError, lambda: t.reorder(i32([[0, 0]]))),
        (ValueError, lambda: t.reorder(i32([[0, 0], [0, 0]]), wg.KvPlanes([torch.zeros((16, 8, 2), device="cuda")], 8))),
        (ValueError, lambda: t.reorder(i32([[0, 0], [0, 0]]), wg.KvPlanes([torch.zeros((15, 4, 2), device="cuda")], 4))),
        (ValueError, lambda: wg.KvPlanes([torch.zeros((16, 8, 2), device="cuda")], 4)),
        (ValueError, lambda: wg.KvPlanes([torch.zeros((16, 4, 2))], 4)),
        (ValueError, lambda: wg.KvPlanes([], 4)),
        (ValueError, lambda: pool.load(i32([0] * 15))),
    ]
    for error, call in cases:
        with pytest.raises(error):
            call()
    lib, p = wg.binding._lib, table.data_ptr()
    h = pool.handle
    assert lib.wg_kv_extend(None, p, 5, 5, p, p, 4, p, p, p, p, 1, None, None) == -1
    assert lib.wg_kv_extend(h, p, 4, 5, p, p, 4, p, p, p, p, 1, None, None) == -1      # stride below max_blocks
    assert lib.wg_kv_extend(h, p, 5, 5, p, p, 5, p, p, p, p, 1, None, None) == -1      # beyond max_seqs
    assert lib.wg_kv_extend(h, p, 5, 5, p, p, 4, p, None, p, p, 1, None, None) == -1
    assert lib.wg_kv_extend(h, p, 5, 5, p, p, 4, p, p, p, p, -1, None, None) == -1
    assert lib.wg_kv_shrink(h, p, 5, 5, p, None, 4, None, None) == -1
    assert lib.wg_kv_shrink(h, p, 5, 0, p, p, 4, None, None) == -1
    assert lib.wg_kv_reorder(h, p, 5, 5, p, p, 1, 33, None, 0, None, None, None, None) == -1
    assert lib.wg_kv_reorder(h, p, 5, 5, p, p, 2, 4, None, 0, None, None, None, None) == -1
    assert lib.wg_kv_reorder(h, p, 5, 5, p, p, 1, 4, None, 2, None, None, None, None) == -1
    assert lib.wg_kv_pool_load(h, None, None) == -1 and lib.wg_kv_pool_refs(None) is None
    torch.cuda.synchronize()
    assert pool.n_free() == 16 and (table == -1).all()
