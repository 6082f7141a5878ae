"""Attention of tokens at the last positions that a length can count: tiles that pass 2^31 with their end."""
import math

import pytest
import torch

import cache_ref as ref

pytestmark = pytest.mark.gpu
BF16, FP16, E4M3, INT8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8
BLOCK, MOST, H, D, ROWS = 1 << 20, 2 ** 31 - 1, 1, 16, 4


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


@pytest.mark.parametrize("held", [BF16, INT8])
@pytest.mark.parametrize("lens", [[MOST], [MOST, MOST - 20, MOST - 40, 5], [MOST - 1, MOST]])
@pytest.mark.parametrize("window", [100, 0])
def test_the_last_positions_of_all(wg, held, lens, window):
    """Only the last block of a table of 2048 is one: all before it are passed over."""
    g, S = ref.generator(1), len(lens)
    values = [torch.randn((1, BLOCK, H, D), generator=g) for _ in range(2)]
    if held is INT8:
        (k, ks), (v, vs) = (ref.codes_of(x, held) for x in values)
        cache = wg.KvCache(*(x.cuda() for x in (k, v, ks, vs)))
    else:
        (k, v), ks, vs = (x.to(held) for x in values), None, None
        cache = wg.KvCache(k.cuda(), v.cuda())
    pool = wg.KvPool(1, BLOCK, S)
    table = torch.full((S, (MOST + 1) // BLOCK), -1, dtype=torch.int32)
    table[:, -1] = 0
    tables = wg.KvTables(pool, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = torch.randn((S, ROWS, D), generator=g).to(BF16)
    k, v = ref.held(k, ks)[0, :, 0], ref.held(v, vs)[0, :, 0]
    attend = wg.Attend(S, ROWS, H, D)
    for group in (1, S):
        out, lse = torch.full((S, ROWS, D), 7.0, dtype=BF16, device="cuda"), torch.full((S, ROWS), 7.0, device="cuda")
        attend(q.cuda(), cache, tables, out, lse=lse, window=window, group=group)
        for s, n in enumerate(lens):
            last = n - (MOST + 1 - BLOCK)
            if last <= 0:
                assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
                continue
            first = max(0, last - window) if window else 0
            x = q[s].double() @ k[first:last].T / D ** 0.5
            want, w = torch.logsumexp(x, 1), torch.softmax(x, 1)
            # 2^20 scores of sums of 16 products, each off by a step of 2^-23 at their size, weights in 16 bits, sums of some thousand
            # terms at a time
            off = (x.abs().max() * 4 + 4) * 32 * 2.0 ** -23 + 4000 * 2.0 ** -23
            mean, mass = w @ v[first:last], w @ v[first:last].abs()
            assert ((lse[s].cpu().double() - want).abs() <= off).all()
            assert ((out[s].cpu().double() - mean).abs() <= mean.abs() * 2.0 ** -8 + mass * (2.0 ** -8 + 2 * off)).all()
