"""A NaN among the logits that the denominator covers ends its row, wherever it is and whatever surrounds it: also where
its neighbours are masked, -inf or NaN themselves."""
import numpy as np
import pytest

import beam_ref as ref
from test_gpu_beam import as_dtype, check, make, run, separate

pytestmark = pytest.mark.gpu
V = 6201                       # rows begin at odd places; four steps of a scan in bf16, seven in fp32
PLACES = [0, 1, 1023, 1024, 2047, 2048, 3000, 4095, 4096, 6100, V - 1]
NORMS = [ref.NORM_ALLOWED, ref.NORM_FULL]


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def same(wg, x, allowed, score, norm, n_req, n_out, rng, dtype):
    t = as_dtype(x, dtype)
    xf = t.float().numpy()
    rows = len(x)
    score = separate(xf, allowed, score, np.zeros(rows, bool), 0, norm, n_req, n_out, rng)
    want = ref.select(xf, allowed, score, np.zeros(rows, bool), 0, norm, n_req, n_out)
    check(run(wg, t, allowed, score, None, 0, norm, n_req, n_out), want)
    return want


def batch(dtype, n_req, K, seed):
    rng = np.random.default_rng(seed)
    x, _, _, score, _, _ = make(seed, n_req, K, V, dtype, "all", ref.NORM_NONE, 2, dead=False)
    return rng, x.float().numpy().copy(), score


# one launch, and two
@pytest.mark.parametrize("n_req,K", [(1, 2), (3, 4), (160, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", NORMS)
def test_an_allowed_nan_alone_in_its_step(wg, n_req, K, dtype, norm):
    """Two allowed tokens, far apart, one of them NaN, in every other row."""
    for at in PLACES:
        rng, x, score = batch(dtype, n_req, K, at)
        allowed = np.zeros(x.shape, bool)
        other = (at + V // 2) % V
        allowed[:, [at, other]] = True
        x[::2, at] = np.nan
        want = same(wg, x, allowed, score, norm, n_req, 2, rng, dtype)
        assert all(b % 2 == 1 for line in want for _, b, _ in line)


@pytest.mark.parametrize("n_req,K", [(1, 2), (160, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", NORMS)
@pytest.mark.parametrize("around", [np.nan, -np.inf])
def test_steps_of_nothing_else(wg, n_req, K, dtype, norm, around):
    """Slices of the vocabulary that are NaN or -inf through and through, one NaN at least among them."""
    for begin, end, at in ((0, 2100, 5), (0, 2100, 2099), (2040, 4200, 2047), (2040, 4200, 4100), (4090, V, V - 1), (0, V, 3333)):
        rng, x, score = batch(dtype, n_req, K, begin + at)
        x[::2, begin:end] = around
        x[::2, at] = np.nan
        allowed = rng.random(x.shape) < 0.9
        allowed[:, at] = True
        want = same(wg, x, allowed, score, norm, n_req, 2, rng, dtype)
        assert all(b % 2 == 1 for line in want for _, b, _ in line)


@pytest.mark.parametrize("n_req,K", [(1, 2), (160, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_masked_nan_in_a_step_of_nothing_else(wg, n_req, K, dtype):
    """Masked NaN are no part of the allowed tokens' denominator, and are of the whole vocabulary's."""
    for begin, end in ((0, 2100), (2040, 4200), (4090, V)):
        rng, x, score = batch(dtype, n_req, K, begin)
        x[:, begin:end] = -np.inf
        x[::2, begin + 7:end:5] = np.nan
        allowed = rng.random(x.shape) < 0.9
        allowed[:, begin + 7:end:5] = False
        same(wg, x, allowed, score, ref.NORM_ALLOWED, n_req, 2, rng, dtype)
        assert len(ref.row_scores(x[0], allowed[0], 0.0, False, 0, ref.NORM_ALLOWED)[0])
        want = same(wg, x, allowed, score, ref.NORM_FULL, n_req, 2, rng, dtype)
        assert all(b % 2 == 1 for line in want for _, b, _ in line)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steps_of_minus_infinity_are_no_nan(wg, dtype):
    rng, x, score = batch(dtype, 2, 4, 3)
    for row, (begin, end) in enumerate([(0, 2100), (2040, 4200), (4090, V), (1, V), (0, V - 1), (0, V), (100, 101), (0, 1)]):
        x[row, begin:end] = -np.inf
    for norm in (*NORMS, ref.NORM_NONE):
        same(wg, x, np.ones(x.shape, bool), score, norm, 2, 2, rng, dtype)
        same(wg, x, rng.random(x.shape) < 0.5, score, norm, 2, 2, rng, dtype)
