"""MXFP4 quantisation and product on the GPU against 64-bit restatements on the CPU."""
import numpy as np
import pytest

from tests import ops_util as ou

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


def quantize(s2d2, x, guard=64):
    """codes, scales (with `guard` untouched bytes behind each) of a 2-d device tensor."""
    name = "fp32" if x.dtype == torch.float32 else "bf16"
    nc, ns = s2d2.mxfp4_sizes(*x.shape)
    codes, scales = (torch.full((n + guard,), 0xA5, dtype=torch.uint8, device="cuda") for n in (nc, ns))
    s2d2.mxfp4_quantize(x.data_ptr(), name, x.shape[0], x.shape[1], x.stride(0), codes.data_ptr(), scales.data_ptr(), stream())
    return codes, scales


def check_codes(x64, codes, scales):
    want_c, want_s = ou.mxfp4_encode(x64)
    want_s = ou.tile_scales(want_s)
    got_c, got_s = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(got_c[:want_c.size].reshape(want_c.shape), want_c)
    assert np.array_equal(got_s[:want_s.size], want_s)
    assert (got_c[want_c.size:] == 0xA5).all() and (got_s[want_s.size:] == 0xA5).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,lead", [(1, 1, 0, 0), (1, 31, 1, 0), (3, 33, 0, 0), (5, 128, 0, 0), (129, 257, 7, 3),
                                                (128, 512, 0, 1), (300, 1000, 24, 8), (1, 4096, 0, 0), (257, 40, 0, 0)])
def test_quantize_and_back(s2d2, dtype, rows, cols, pad, lead):
    """Every code and scale byte, padding too, and the values they stand for; odd strides and unaligned first elements."""
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    buf = torch.randn(rows * (cols + pad) + lead, generator=g, device="cuda")
    buf *= torch.exp(3 * torch.randn(buf.shape, generator=g, device="cuda"))
    x = buf.to(DT[dtype])[lead:].view(rows, cols + pad)[:, :cols]
    codes, scales = quantize(s2d2, x)
    x64 = x.double().cpu().numpy()
    check_codes(x64, codes, scales)
    want = ou.mxfp4_values(*ou.mxfp4_encode(x64), cols)
    for out in ("fp32", "bf16"):
        y = torch.full((rows * (cols + pad) + lead,), 7.0, dtype=DT[out], device="cuda")
        yv = y[lead:].view(rows, cols + pad)
        s2d2.mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), rows, cols, yv.data_ptr(), out, cols + pad, stream())
        assert np.array_equal(yv[:, :cols].double().cpu().numpy(), want)          # exact in both types
        assert (yv[:, cols:] == 7).all() and (y[:lead] == 7).all()


def test_quantize_special_values(s2d2):
    big = np.finfo(np.float32).max
    sub = 2.0 ** -149
    rows = [[6, -6, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -0.75, -5], [7, 7.999, -7.5, 6.001], [0.0, -0.0], [big, -big, big / 8],
            [sub, -sub, 3 * sub], [2.0 ** -126, 2.0 ** -127, -(2.0 ** -128)], [np.inf, 1], [np.nan, 1], [-np.inf, np.nan],
            [1.0, 2.0 ** -30], [2.0 ** -124, 2.0 ** -127, 3 * 2.0 ** -128]]
    x = np.zeros((len(rows), 64), np.float32)
    for i, r in enumerate(rows):
        x[i, :len(r)] = r
        x[i, 40] = 1.0                                                            # a second, ordinary block
    codes, scales = quantize(s2d2, torch.from_numpy(x).cuda())
    check_codes(x.astype(np.float64), codes, scales)
    y = torch.empty(x.shape, device="cuda")
    s2d2.mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), *x.shape, y.data_ptr(), "fp32", 64, stream())
    assert np.array_equal(y.double().cpu().numpy(), ou.mxfp4_values(*ou.mxfp4_encode(x.astype(np.float64)), 64), equal_nan=True)


def operand(rows, K, seed, scale=1.0):
    g = np.random.default_rng(seed)
    x = (g.standard_normal((rows, K)) * np.exp(g.standard_normal((rows, 1)))).astype(np.float32) * np.float32(scale)
    codes, s = ou.mxfp4_encode(x.astype(np.float64))
    return (torch.from_numpy(codes).cuda(), torch.from_numpy(ou.tile_scales(s)).cuda()), ou.mxfp4_values(codes, s, K)


def product_tolerance(xv, wv, scale, y_type):
    """Products of e2m1 codes and powers of two are exact; the sum rounds (or truncates, hence 2^-23) once per 64 elements and a few
    times where k is split; then the scale and y's type."""
    size = (np.abs(xv) @ np.abs(wv).T) * abs(scale)
    y = np.abs(xv @ wv.T) * abs(scale)
    K = xv.shape[1]
    return size * ((K + 63) // 64 + 10) * 2.0 ** -23 + y * (2.0 ** -23 + (2.0 ** -8 if y_type == "bf16" else 0.0)) + 1e-37


SHAPES = [(1, 1, 1), (1, 128, 32), (2, 8, 33), (16, 127, 64), (17, 129, 65), (5, 256, 256), (3, 130, 257), (33, 1000, 512),
          (64, 384, 4096), (1, 4096, 4096), (65, 200, 300), (77, 1001, 2050), (128, 256, 1024), (129, 300, 700), (200, 128, 96),
          (256, 512, 512), (300, 640, 1000), (513, 257, 288),
          # enough tiles for pairs of CTAs: one or several tiles per pair, every tile width and start inside a scale tile
          (150, 9500, 96), (300, 6001, 320), (1000, 2500, 257), (1025, 2999, 64), (210, 19000, 600), (450, 10000, 1024),
          (1400, 1537, 1000)]


@pytest.mark.parametrize("y_type", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(s2d2, M, N, K, y_type):
    (xc, xs), xv = operand(M, K, M * 7 + K)
    (wc, ws), wv = operand(N, K, N * 3 + K, 0.02)
    pad, scale = 5, 0.75
    y = torch.full((M + 1, N + pad), 7.0, dtype=DT[y_type], device="cuda")
    s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), y_type, M, N, K, N + pad, scale, stream())
    s2d2.ops_status(stream())
    got = y.double().cpu().numpy()
    want = scale * (xv @ wv.T)
    err, tol = np.abs(got[:M, :N] - want), product_tolerance(xv, wv, scale, y_type)
    assert np.isfinite(got).all() and (err <= tol).all(), (err.max(), (err / tol).max())
    assert (got[:M, N:] == 7).all() and (got[M:] == 7).all()


def test_product_of_head_rows(s2d2):
    """A head of 100 000 rows: more tiles than CTAs fit at once; a sample of the columns is checked."""
    M, N, K = 3, 100000, 512
    g = torch.Generator(device="cuda").manual_seed(1)
    w = torch.randn(N, K, generator=g, device="cuda") * 0.02
    wc, ws = quantize(s2d2, w, 0)
    (xc, xs), xv = operand(M, K, 5)
    y = torch.empty(M, N, device="cuda")
    s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
    s2d2.ops_status(stream())
    at = np.r_[0:200, 50000:50200, N - 200:N]
    wv = ou.mxfp4_values(*ou.mxfp4_encode(w[at].double().cpu().numpy()), K)
    err = np.abs(y[:, at].double().cpu().numpy() - xv @ wv.T)
    assert (err <= product_tolerance(xv, wv, 1.0, "fp32")).all()


@pytest.mark.parametrize("M", [3, 200])
def test_nan_blocks_stay_in_their_rows(s2d2, M):
    N, K = 140, 192
    g = np.random.default_rng(9)
    x, w = g.standard_normal((M, K)).astype(np.float32), g.standard_normal((N, K)).astype(np.float32)
    x[1, 70], w[130, 5] = np.nan, np.inf
    xc, xs = quantize(s2d2, torch.from_numpy(x).cuda(), 0)
    wc, ws = quantize(s2d2, torch.from_numpy(w).cuda(), 0)
    y = torch.empty(M, N, device="cuda")
    s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
    bad = np.zeros((M, N), bool)
    bad[1], bad[:, 130] = True, True
    assert np.array_equal(np.isnan(y.cpu().numpy()), bad)


def test_empty_batch_and_bad_pointers(s2d2):
    y = torch.full((4,), 7.0, device="cuda")
    s2d2.mxfp4_gemm(0, 0, 0, 0, 0, "fp32", 0, 4, 32, stream=stream())
    s2d2.mxfp4_quantize(0, "fp32", 0, 32, 32, 0, 0, stream())
    host = torch.zeros(64)
    q = torch.zeros(1024, dtype=torch.uint8, device="cuda")
    for args in [(0, q.data_ptr(), q.data_ptr()), (y.data_ptr(), 0, q.data_ptr()), (y.data_ptr(), q.data_ptr() + 8, q.data_ptr()),
                 (host.data_ptr(), q.data_ptr(), q.data_ptr()), (y.data_ptr() + 2, q.data_ptr(), q.data_ptr())]:
        with pytest.raises(s2d2.S2D2Error) as e:
            s2d2.mxfp4_quantize(args[0], "fp32", 1, 4, 4, args[1], args[2], stream())
        assert e.value.code == -1
    assert (y == 7).all()


def test_repeated_calls_agree_bit_for_bit(s2d2):
    for M, N, K in [(1, 640, 4096), (40, 300, 2048), (300, 640, 1024)]:
        (xc, xs), _ = operand(M, K, 1)
        (wc, ws), _ = operand(N, K, 2)
        ys = [torch.empty(M, N, device="cuda") for _ in range(4)]
        for y in ys:
            s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
        assert all(torch.equal(ys[0], y) for y in ys[1:])


def test_captured_and_concurrent_calls(s2d2):
    """quantise + product in two captured graphs, replayed on two streams at a time with new inputs: nothing is shared."""
    N, K = 384, 2048
    w = torch.randn(N, K, device="cuda") * 0.05
    wc, ws = quantize(s2d2, w, 0)
    wv = ou.mxfp4_values(*ou.mxfp4_encode(w.double().cpu().numpy()), K)
    graphs = []
    for M in (9, 260):
        x = torch.zeros(M, K, device="cuda")
        nc, ns = s2d2.mxfp4_sizes(M, K)
        xc, xs = torch.empty(nc, dtype=torch.uint8, device="cuda"), torch.empty(ns, dtype=torch.uint8, device="cuda")
        y = torch.empty(M, N, device="cuda")

        def call():
            s2d2.mxfp4_quantize(x.data_ptr(), "fp32", M, K, K, xc.data_ptr(), xs.data_ptr(), stream())
            s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())

        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append((g, x, y, M, (xc, xs), torch.cuda.Stream()))
    for trial in range(3):
        for g, x, y, M, _, st in graphs:
            x.copy_(torch.randn(M, K, generator=torch.Generator().manual_seed(trial * 10 + M)))
        torch.cuda.synchronize()
        for g, x, y, M, _, st in graphs:
            with torch.cuda.stream(st):
                for _ in range(3):
                    g.replay()
        torch.cuda.synchronize()
        for g, x, y, M, _, st in graphs:
            xv = ou.mxfp4_values(*ou.mxfp4_encode(x.double().cpu().numpy()), K)
            err = np.abs(y.double().cpu().numpy() - xv @ wv.T)
            assert (err <= product_tolerance(xv, wv, 1.0, "fp32")).all()


@pytest.mark.parametrize("M,N,K", [(1, 1000000, 64), (40000, 300, 32), (6, 200, 60000), (5000, 5000, 40)])
def test_long_axes(s2d2, M, N, K):
    """Each axis long; a sample of rows and columns is checked."""
    g = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda") * 0.1
    (xc, xs), (wc, ws) = quantize(s2d2, x, 0), quantize(s2d2, w, 0)
    y = torch.full((M, N), float("nan"), device="cuda")
    s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
    s2d2.ops_status(stream())
    assert torch.isfinite(y).all()
    r = np.unique(np.r_[0:min(M, 40), M // 2:min(M, M // 2 + 40), max(0, M - 40):M])
    c = np.unique(np.r_[0:min(N, 150), N // 2:min(N, N // 2 + 150), max(0, N - 150):N])
    xv = ou.mxfp4_values(*ou.mxfp4_encode(x[r].double().cpu().numpy()), K)
    wv = ou.mxfp4_values(*ou.mxfp4_encode(w[c].double().cpu().numpy()), K)
    err = np.abs(y[r][:, c].double().cpu().numpy() - xv @ wv.T)
    assert (err <= product_tolerance(xv, wv, 1.0, "fp32")).all()


def test_the_largest_axes(s2d2):
    """Columns and K, and rows, at their documented limits; a sample is checked."""
    K, M, N = 1048576, 3, 140
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda") * 0.1
    (xc, xs), (wc, ws) = quantize(s2d2, x, 0), quantize(s2d2, w, 0)
    y = torch.empty(M, N, device="cuda")
    s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, N, K, stream=stream())
    s2d2.ops_status(stream())
    xv = ou.mxfp4_values(*ou.mxfp4_encode(x.double().cpu().numpy()), K)
    c = [0, 1, 127, 128, N - 1]
    wv = ou.mxfp4_values(*ou.mxfp4_encode(w[c].double().cpu().numpy()), K)
    err = np.abs(y[:, c].double().cpu().numpy() - xv @ wv.T)
    assert (err <= product_tolerance(xv, wv, 1.0, "fp32")).all()
    del x, w, xc, xs, wc, ws
    rows = 4194304
    x = torch.randn(rows, 3, generator=g, device="cuda")
    codes, scales = quantize(s2d2, x, 0)
    back = torch.empty_like(x)
    s2d2.mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), rows, 3, back.data_ptr(), "fp32", 3, stream())
    at = np.r_[0:300, rows // 2:rows // 2 + 300, rows - 300:rows]
    want = ou.mxfp4_values(*ou.mxfp4_encode(x[at].double().cpu().numpy()), 3)
    assert np.array_equal(back[at].double().cpu().numpy(), want)


def test_calls_from_several_host_threads(s2d2):
    """Threads with streams of their own: results as alone, and each thread reads the text of its own failure."""
    import threading
    K = 1024
    (wc, ws), wv = operand(600, K, 11)
    jobs = [operand(M, K, M) for M in (1, 40, 130, 300)]
    failures, outs = [], {}

    def work(i):
        try:
            (xc, xs), xv = jobs[i]
            M = xv.shape[0]
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                y = torch.empty(M, 600, device="cuda")
                for _ in range(20):
                    s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, 600, K,
                                    stream=st.cuda_stream)
                    try:
                        s2d2.mxfp4_gemm(xc.data_ptr(), xs.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "fp32", M, 600, K,
                                        y_stride=i, stream=st.cuda_stream) if i % 2 else s2d2.score_logits(y.data_ptr(), "fp32", M, 0, 600)
                    except s2d2.S2D2Error as e:
                        assert ("y_stride" if i % 2 else "vocab") in str(e), str(e)
                st.synchronize()
                outs[i] = y
        except BaseException as e:      # noqa: BLE001 - reported below
            failures.append(repr(e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    for i, (_, xv) in enumerate(jobs):
        assert (np.abs(outs[i].double().cpu().numpy() - xv @ wv.T) <= product_tolerance(xv, wv, 1.0, "fp32")).all()


def test_rows_further_apart_than_32_bits(s2d2):
    """Inputs and outputs whose rows lie 2^31 + 8 elements apart: offsets of the last row pass 2^32."""
    stride, K, N = 2 ** 31 + 8, 200, 130
    buf = torch.empty(2 * stride + K, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, K), (stride, 1))
    x.copy_(torch.randn(3, K, generator=torch.Generator().manual_seed(1)))
    codes, scales = quantize(s2d2, x)
    check_codes(x.double().cpu().numpy(), codes, scales)
    want = ou.mxfp4_values(*ou.mxfp4_encode(x.double().cpu().numpy()), K)
    buf.zero_()
    s2d2.mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), 3, K, buf.data_ptr(), "bf16", stride, stream())
    assert np.array_equal(x.double().cpu().numpy(), want)
    (wc, ws), wv = operand(N, K, 2)
    y = torch.as_strided(buf, (3, N), (stride, 1))
    s2d2.mxfp4_gemm(codes.data_ptr(), scales.data_ptr(), wc.data_ptr(), ws.data_ptr(), y.data_ptr(), "bf16", 3, N, K, stride, stream=stream())
    s2d2.ops_status(stream())
    assert (np.abs(y.double().cpu().numpy() - want @ wv.T) <= product_tolerance(want, wv, 1.0, "bf16")).all()


FIRST_USE = """
import sys, torch
import paper_2603_25702_b200 as s
torch.cuda.set_device(0)
st = torch.cuda.Stream()
M, N, K = 300, 20000, 256
x, w = torch.randn(M, K, device="cuda"), torch.randn(N, K, device="cuda")
bufs = [[torch.empty(n, dtype=torch.uint8, device="cuda") for n in s.mxfp4_sizes(*t.shape)] for t in (x, w)]
y, lse = torch.empty(M, N, device="cuda"), torch.empty(2, M, device="cuda")
tok = torch.zeros(M, dtype=torch.int32, device="cuda")
ws = torch.empty(s.mxfp4_score_workspace(M, N, K), dtype=torch.uint8, device="cuda")
torch.cuda.synchronize()
with torch.cuda.stream(st):
    s.ops_status(st.cuda_stream)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        p = [b.data_ptr() for pair in bufs for b in pair]
        for t, (c, sc) in zip((x, w), bufs):
            s.mxfp4_quantize(t.data_ptr(), "fp32", t.shape[0], K, K, c.data_ptr(), sc.data_ptr(), st.cuda_stream)
        s.mxfp4_gemm(*p, y.data_ptr(), "fp32", M, N, K, stream=st.cuda_stream)
        s.score_logits(y.data_ptr(), "fp32", M, N, N, d_lse=lse[0].data_ptr(), stream=st.cuda_stream)
        s.mxfp4_score(*p, M, N, K, tok.data_ptr(), ws.data_ptr(), ws.numel(), d_lse=lse[1].data_ptr(), stream=st.cuda_stream)
    g.replay()
    s.ops_status(st.cuda_stream)
want = torch.logsumexp(y.double(), 1)
assert (lse[0] - want).abs().max() < 1e-3 and (lse[1] - want).abs().max() < 1e-3, (lse, want)
print("captured first use ok")
"""


def test_first_use_may_be_captured_after_ops_status():
    """In a fresh process: s2d2_ops_status loads every kernel, then the first launches happen inside a capture."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_USE], cwd=root, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and "captured first use ok" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
