"""Scores from hidden rows at the ends of fp32's range and with logits that are not finite."""
import numpy as np
import pytest

from tests import ops_util as ou
from tests.test_gpu_mxfp4_score import run

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FMAX = float(np.finfo(np.float32).max)
# Error of the log of a sum of exponentials, whatever the number of terms: exponentials 2^-22 and their arguments 2^-23; at most 32 additions
# one after the other (2^-24 each) before a compensated sum takes over; 13 merges of partial sums (each a factor 2^-22 and two
# roundings); factors where the reference of the exponentials rises, the k-th last of them weighted by e^-k.  6.5e-6 in all.
SUMS = 2.0 ** -17


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def on_gpu(x64):
    codes, s = ou.mxfp4_encode(x64)
    return (torch.from_numpy(codes).cuda(), torch.from_numpy(ou.tile_scales(s)).cuda()), ou.mxfp4_values(codes, s, x64.shape[1])


def check(got, want):
    """`want` as ops_util.scores returns it for logits that are exact in fp32."""
    t = SUMS + want["log_s"] * 2.0 ** -22
    for n, g, tol in (("logprob", got[0], t), ("lse", got[1], t), ("entropy", got[2], 3 * t * (1 + np.nan_to_num(want["entropy"])))):
        w = np.where(want[n] < -FMAX, -np.inf, want[n])
        assert np.array_equal(np.isnan(w), np.isnan(g)), (n, w, g)
        fine = np.isfinite(w)
        assert np.array_equal(w[~fine & ~np.isnan(w)], g[~fine & ~np.isnan(w)]), (n, w, g)
        err = np.abs(np.where(fine, g, 0) - np.where(fine, w, 0))
        assert (err <= tol + 2.0 ** -22 * np.abs(np.where(fine, w, 0))).all(), (n, err.max(), w[err.argmax()], g[err.argmax()])
    e = got[2][~np.isnan(got[2])]
    assert (e >= 0).all()


@pytest.mark.parametrize("N", [1000, 8])
@pytest.mark.parametrize("M", [40, 170])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** 30, -(2.0 ** 30), 1.1e9])
def test_ends_of_the_range(s2d2, M, N, scale):
    """Logits up to 2.55e38 and -2.55e38, differences beyond fp32, and infinities of either sign in one place of a row."""
    unit = 1.5 * 2.0 ** 40
    w = np.zeros((N, 64))
    first, last = N // 2, N - 1
    w[:, 0] = -unit
    w[[1, first], 0] = unit                          # two large ones, all others small
    w[:, 1] = 0.0
    w[1, 1] = -unit                                  # one small one
    w[last, 2] = -unit                               # one small one in the last columns
    w[first, 3] = unit                               # one large one
    # x times the unit times |scale|: 1.28e38, 2.55e38, infinite, ordinary
    sizes = np.array([2.0 ** 86, 2.0 ** 87, 2.0 ** 100, 2.0 ** -40]) / abs(scale)
    x = np.zeros((M, 64))
    for r in range(M):
        if r % 17 < 16:
            x[r, (r % 17) // 4] = sizes[r % 4] * (1.0 if r < M // 2 else -1.0)
    (xg, xv), (wg, wv) = on_gpu(x), on_gpu(w)
    with np.errstate(over="ignore"):
        logits = (float(np.float32(scale)) * (xv @ wv.T)).astype(np.float32).astype(np.float64)     # exact products, rounded once
    tokens = np.array([1, first, last, 0])[np.arange(M) // 3 % 4]
    want = ou.scores(logits, tokens)
    bad = ~np.isfinite(logits).all(axis=1)
    assert bad.any() and not bad.all()
    for n in ("logprob", "lse", "entropy"):
        want[n][bad] = np.nan
    check(run(s2d2, xg, wg, M, N, 64, tokens, scale), want)


def test_infinite_accumulators(s2d2):
    """Products that overflow before `scale` brings them back: such a row is NaN, the others are as they should be."""
    M, N = 200, 300
    w = np.zeros((N, 32))
    w[7, 0], w[:, 1] = -(2.0 ** 100), 1.0
    x = np.zeros((M, 32))
    x[:, 1] = np.arange(M) % 5
    x[3::7] = 0
    x[3::7, 0] = 2.0 ** 100
    # (the head's row 7 keeps nothing beside 2^100)
    (xg, xv), (wg, wv) = on_gpu(x), on_gpu(w)
    want = ou.scores(2.0 ** -90 * (xv @ wv.T), np.zeros(M, int))
    for n in ("logprob", "lse", "entropy"):
        want[n][3::7] = np.nan
    check(run(s2d2, xg, wg, M, N, 32, np.zeros(M, int), 2.0 ** -90), want)
