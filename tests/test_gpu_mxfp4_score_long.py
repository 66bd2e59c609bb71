"""Scores from hidden rows over the longest heads: the error does not grow with the number of logits."""
import numpy as np
import pytest

from tests import ops_util as ou
from tests.test_gpu_mxfp4_score import run
from tests.test_gpu_mxfp4_score_range import SUMS, check, on_gpu

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


LONG_M = 40961      # so many rows that one cluster takes the whole head for each of them


def test_longest_head_rising_and_falling(s2d2):
    """Logits slope * n over 4194304 head rows: the digits of n to the base 4 stand in blocks of their own."""
    N, blocks = 4194304, 11
    K = blocks * 32
    n = torch.arange(N, device="cuda")
    codes = torch.zeros(N, blocks, 16, dtype=torch.uint8, device="cuda")
    e2m1 = torch.tensor([0, 2, 4, 5], dtype=torch.uint8, device="cuda")                  # 0, 1, 2, 3
    for d in range(blocks):
        codes[:, d, 0] = e2m1[n // 4 ** d % 4]
    tile = torch.full((3, 512), 127, dtype=torch.uint8, device="cuda")
    tile[2, 3::4] = 0                                                                    # there is no twelfth block
    w = (codes.view(-1), tile.repeat(N // 128, 1, 1).view(-1))
    slopes = [2.0 ** -16, 2.0 ** -18, 2.0 ** -20, 2.0 ** -23, -(2.0 ** -18), -(2.0 ** -20), 0.0]
    x = np.zeros((len(slopes), K))
    for d in range(blocks):
        x[:, 32 * d] = np.array(slopes) * 4.0 ** d
    xc, xs = ou.mxfp4_encode(x)
    assert np.array_equal(ou.mxfp4_values(xc, xs, K), x)
    row = np.arange(LONG_M) % len(slopes)
    xg = (torch.from_numpy(xc[row]).cuda(), torch.from_numpy(ou.tile_scales(xs[row])).cuda())
    tokens = (np.arange(LONG_M, dtype=np.int64) * 1048583) % N
    got = run(s2d2, xg, w, LONG_M, N, K, tokens)
    want = {k: np.zeros(LONG_M) for k in ("logprob", "lse", "entropy", "log_s")}
    for i, slope in enumerate(slopes):
        one = ou.scores(slope * np.arange(N, dtype=np.float64)[None], [0])
        at = np.arange(i, LONG_M, len(slopes))
        want["lse"][at], want["entropy"][at], want["log_s"][at] = one["lse"][0], one["entropy"][0], one["log_s"][0]
        want["logprob"][at] = slope * tokens[at] - one["lse"][0]
    check(got, want)


@pytest.mark.parametrize("N", [151936, 4194304])
def test_many_rows_against_long_heads(s2d2, N):
    """Random logits, and logits that are all equal but for a few: small terms next to a large sum.  The head repeats itself."""
    K, period = 32, {151936: 151936 // 8, 4194304: 32768}[N]
    if period % 128:
        period = N // 1187                                                               # 128 rows: scale tiles repeat as a whole
    g = np.random.default_rng(N)
    w = g.standard_normal((period, K)) * 2.5 / K ** 0.5
    w[:, 31], w[0, 31] = 0.5, 1.0
    codes, s = ou.mxfp4_encode(w)
    wv, times = ou.mxfp4_values(codes, s, K), N // period
    wg = (torch.from_numpy(codes).cuda().repeat(times, 1).view(-1), torch.from_numpy(ou.tile_scales(s)).cuda().repeat(times))
    x = g.standard_normal((LONG_M, K))
    x[1::3] = 0
    x[1::3, 31] = g.uniform(0.3, 3, x[1::3, 31].shape)
    xg, xv = on_gpu(x)
    tokens = g.integers(0, N, LONG_M)
    got = run(s2d2, xg, wg, LONG_M, N, K, tokens)
    at = np.unique(np.r_[0:40, 20000:20040, LONG_M - 40:LONG_M])
    want = ou.scores(xv[at] @ wv.T, tokens[at] % period)
    more = np.log(times)
    for n, sign in (("lse", 1), ("entropy", 1), ("log_s", 1), ("logprob", -1)):
        want[n] += sign * more
    # a logit is off by at most `slack` (one rounding or truncation of the sum, one of the scale's product)
    slack = ((np.abs(xv[at]) @ np.abs(wv).T) * 3 * 2.0 ** -23).max()
    t = SUMS + want["log_s"] * 2.0 ** -22 + 2.0 ** -22 * np.abs(want["lse"])
    spread = np.ptp(xv[at] @ wv.T, axis=1)
    for n, row, tol in (("logprob", 0, t + 2 * slack + 2.0 ** -22 * np.abs(want["logprob"])), ("lse", 1, t + slack),
                        ("entropy", 2, 3 * t * (1 + want["entropy"]) + 2 * slack * (1 + spread))):
        err = np.abs(got[row][at] - want[n])
        assert (err <= tol).all(), (n, err.max(), (err / tol).max())
