"""Logits far from zero: finite values that stand for a mask (-1e9, -1e10, ...), and whatever else a model may put out.

Tolerance, derived before the first run: as in test_gpu_beam, 2^-16 + 4 * M * 2^-23 with M the largest size
among score, logits and lse that take part.
"""
import numpy as np
import pytest

import beam_ref as ref
from test_gpu_beam import as_dtype, check, run

pytestmark = pytest.mark.gpu
SIZES = [1e3, 1e5, 2.0 ** 20 - 1, 2.0 ** 20, 3e7, 1e9, 2e9, 1e10, 1e12, 1e15, 1e20, 1e30, 3e38]


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def same(wg, x, allowed, norm, dtype, n_out=4):
    """Every row a request of its own, by itself (one launch) and in a batch of many (two)."""
    t = as_dtype(x, dtype)
    xf = t.float().numpy()
    n = len(x)
    score = -np.arange(n, dtype=np.float32) / 8
    want = ref.select(xf, allowed, score, np.zeros(n, bool), 0, norm, n, n_out)
    times = -(-200 // n)
    for k in (1, times):
        rep = lambda a: np.concatenate([a] * k)  # noqa: E731
        got = run(wg, t.repeat(k, 1), rep(allowed), rep(score), None, 0, norm, n * k, n_out)
        for r, line in enumerate(want * k):
            one = tuple(g[r:r + 1] for g in got)
            assert len(line) == n_out
            most = np.abs(xf[r % n][[t for _, _, t in line]]).max()
            check(one, [line], 2.0 ** -16 + 4 * max(most, 64) * 2.0 ** -23)


def rows_around(sizes, V, sign):
    """Rows whose logits are 1, 127/128, ... of a size (steps that bf16 can tell apart); the four largest differ."""
    x = np.zeros((len(sizes), V), np.float64)
    rng = np.random.default_rng(V)
    for i, size in enumerate(sizes):
        k = rng.integers(8, 64, V)
        k[rng.permutation(V)[:4]] = [0, 2, 4, 6]
        x[i] = sign * size * (1 - sign * k / 128)
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [ref.NORM_ALLOWED, ref.NORM_FULL])
@pytest.mark.parametrize("V", [40, 5000])
@pytest.mark.parametrize("sign", [1, -1])
def test_rows_of_one_size(wg, dtype, norm, V, sign):
    x = rows_around(SIZES[:-1], V, sign)
    same(wg, x, np.ones(x.shape, bool), norm, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [ref.NORM_ALLOWED, ref.NORM_FULL])
def test_finite_masks_beside_logits(wg, dtype, norm):
    """Most of a row at a large negative value, whole steps of it, and a few logits beside it."""
    V = 6000
    rng = np.random.default_rng(1)
    x = np.repeat(-np.array(SIZES)[:, None], V, 1)
    few = rng.permutation(V)[:6]
    x[:, few] = np.arange(6) * 0.75 - 2
    same(wg, x, np.ones(x.shape, bool), norm, dtype)
    x[:, 2500:2506] = np.arange(6) * 0.75 + 3
    same(wg, x, np.ones(x.shape, bool), norm, dtype)


def test_steps_on_both_sides_of_any_limit(wg):
    """Steps whose maxima lie close together, around every power of two."""
    V = 4096
    x = np.full((26, V), -np.inf)
    for i in range(26):
        size = 2.0 ** (i + 6)
        x[i, [10, 1500, 2600, 4000]] = size * (1 + np.array([-1, -0.5, 0.25, 0.75]) * 2.0 ** -20)
    same(wg, x, np.ones(x.shape, bool), ref.NORM_ALLOWED, "fp32")
