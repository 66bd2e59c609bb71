"""Token scores straight from MXFP4 hidden rows and an MXFP4 head against a 64-bit restatement on the CPU."""
import numpy as np
import pytest

from tests import ops_util as ou

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


def operand(rows, K, seed, size=1.0):
    g = np.random.default_rng(seed)
    codes, s = ou.mxfp4_encode(g.standard_normal((rows, K)) * size)
    return (torch.from_numpy(codes).cuda(), torch.from_numpy(ou.tile_scales(s)).cuda()), ou.mxfp4_values(codes, s, K)


def call(s2d2, x, w, M, N, K, tokens, scale, out, ws):
    s2d2.mxfp4_score(x[0].data_ptr(), x[1].data_ptr(), w[0].data_ptr(), w[1].data_ptr(), M, N, K, tokens.data_ptr(), ws.data_ptr(),
                     ws.numel(), scale=scale, d_logprob=out[0].data_ptr(), d_lse=out[1].data_ptr(), d_entropy=out[2].data_ptr(),
                     stream=stream())


def run(s2d2, x, w, M, N, K, tokens, scale=1.0):
    out = torch.full((3, M + 1), 7.0, device="cuda")
    ws = torch.full((s2d2.mxfp4_score_workspace(M, N, K) + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    tok = torch.as_tensor(np.asarray(tokens), dtype=torch.int32, device="cuda")
    call(s2d2, x, w, M, N, K, tok, scale, out, ws[:-64])
    s2d2.ops_status(stream())
    assert (out[:, M:] == 7).all() and (ws[-64:] == 0xA5).all()
    return out[:, :M].cpu().numpy().astype(np.float64)


def check(got, xv, wv, tokens, scale):
    """A logit is off by at most `slack` (one rounding or truncation per 64 elements, two more for the scale and the change to
    base 2), so lse is too and a log probability by twice that; entropy's derivative is at most its logits' spread.  On top comes the
    arithmetic of the sums: 32 terms per rescale, up to N / ranges terms in one thread, hence the same form as for logits in memory."""
    x = scale * (xv @ wv.T)
    N, K = wv.shape
    want = ou.scores(x, tokens)
    slack = (np.abs(scale) * (np.abs(xv) @ np.abs(wv).T) * (K // 64 + 12) * 2.0 ** -23).max(axis=1)
    sums = (2 * 32 * (N // 32 + 1) ** 0.5 + 64 + N / 64) * 2.0 ** -24 + 2.0 ** -21 + want["log_s"] * 2.0 ** -22
    spread = x.max(axis=1) - x.min(axis=1)
    for n, g, t in (("logprob", got[0], 2 * slack + sums), ("lse", got[1], slack + sums), ("entropy", got[2], 2 * slack * (1 + spread) + 3 * sums * (1 + want["entropy"]))):
        w = want[n]
        assert np.array_equal(np.isnan(w), np.isnan(g)), n
        err = np.abs(g - w)
        tol = t + 2.0 ** -21 * np.abs(w)
        assert (err[~np.isnan(w)] <= tol[~np.isnan(w)]).all(), (n, np.nanmax(err), np.nanmax(err / tol))


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 31, 33), (2, 1000, 64), (8, 5000, 512), (9, 33, 256), (64, 4097, 300), (127, 257, 96),
                                   (128, 2000, 1024), (129, 2000, 128), (200, 300, 160), (257, 9001, 256), (300, 64, 64), (700, 20000, 64)])
def test_scores_from_hidden_rows(s2d2, M, N, K):
    x, xv = operand(M, K, M + K)
    w, wv = operand(N, K, N + 1, 2.0 / K ** 0.5)
    tokens = np.random.default_rng(M).integers(0, N, M)
    tokens[::3] = (xv @ wv.T).argmax(1)[::3]
    for scale in (1.0, -0.5):
        check(run(s2d2, x, w, M, N, K, tokens, scale), xv, wv, tokens, scale)


def test_many_tokens_per_cluster(s2d2):
    """More row groups than clusters: a cluster takes several, one after the other."""
    M, N, K = 20000, 200, 32
    x, xv = operand(M, K, 1)
    w, wv = operand(N, K, 2, 0.3)
    tokens = np.arange(M) % N
    check(run(s2d2, x, w, M, N, K, tokens), xv, wv, tokens, 1.0)


@pytest.mark.parametrize("M", [5, 150])
def test_tokens_outside_and_rows_that_are_not_finite(s2d2, M):
    N, K = 1000, 128
    g = np.random.default_rng(3)
    xf = g.standard_normal((M, K))
    xf[1, 7] = np.nan
    codes, s = ou.mxfp4_encode(xf)
    x = (torch.from_numpy(codes).cuda(), torch.from_numpy(ou.tile_scales(s)).cuda())
    xv = ou.mxfp4_values(codes, s, K)
    w, wv = operand(N, K, 4, 0.2)
    tokens = np.arange(M) * 3
    tokens[2], tokens[3], tokens[4] = -1, N, 2 ** 31 - 1
    check(run(s2d2, x, w, M, N, K, tokens), xv, wv, tokens, 1.0)


def test_agrees_with_product_and_scores_of_logits(s2d2):
    """The same head through the logits in memory: product, then scores; repeated calls agree bit for bit."""
    M, N, K = 140, 12000, 512
    x, xv = operand(M, K, 1)
    w, wv = operand(N, K, 2, 0.1)
    tok = torch.arange(M, dtype=torch.int32, device="cuda") * 50
    y = torch.empty(M, N, device="cuda")
    s2d2.mxfp4_gemm(x[0].data_ptr(), x[1].data_ptr(), w[0].data_ptr(), w[1].data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
    a = torch.empty(3, M, device="cuda")
    s2d2.score_logits(y.data_ptr(), "fp32", M, N, N, tok.data_ptr(), d_logprob=a[0].data_ptr(), d_lse=a[1].data_ptr(),
                      d_entropy=a[2].data_ptr(), stream=stream())
    ws = torch.empty(s2d2.mxfp4_score_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    outs = [torch.empty(3, M, device="cuda") for _ in range(3)]
    for o in outs:
        call(s2d2, x, w, M, N, K, tok, 1.0, o, ws)
    s2d2.ops_status(stream())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    # both sides sum the same logits in fp32: twice the bound on the sums and a rounding of each logit to base 2
    tol = 2 * ((16 * 3 + 64 + N / 64) * 2.0 ** -24 + 2.0 ** -20) + 2.0 ** -21 * 12
    assert (outs[0] - a).abs().max().item() <= 3 * tol * (1 + a[2].max().item())


def test_captured_calls_with_workspaces_of_their_own(s2d2):
    N, K = 3000, 256
    w, wv = operand(N, K, 2, 0.1)
    runs = []
    for M in (6, 200):
        x, xv = operand(M, K, M)
        tok = torch.arange(M, dtype=torch.int32, device="cuda")
        ws = torch.empty(s2d2.mxfp4_score_workspace(M, N, K), dtype=torch.uint8, device="cuda")
        out = torch.empty(3, M, device="cuda")
        call(s2d2, x, w, M, N, K, tok, 1.0, out, ws)
        torch.cuda.synchronize()
        want = out.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(s2d2, x, w, M, N, K, tok, 1.0, out, ws)
        runs.append((g, out, want, (x, tok, ws), torch.cuda.Stream()))
    for g, out, _, _, _ in runs:
        out.zero_()
    torch.cuda.synchronize()
    for g, out, want, _, st in runs:
        with torch.cuda.stream(st):
            for _ in range(5):
                g.replay()
    torch.cuda.synchronize()
    for g, out, want, _, _ in runs:
        assert torch.equal(out, want)
