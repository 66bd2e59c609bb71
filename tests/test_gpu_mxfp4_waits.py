"""Bounded waits of the MXFP4 products: when they begin, and what a call leaves behind when one runs out."""
import numpy as np
import pytest

from tests import ops_util as ou
from tests.test_gpu_mxfp4 import operand, product_tolerance, stream

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def gemm(s2d2, x, w, y, M, N, K):
    s2d2.mxfp4_gemm(x[0].data_ptr(), x[1].data_ptr(), w[0].data_ptr(), w[1].data_ptr(), y.data_ptr(), "fp32", M, N, K, y.stride(0),
                    stream=stream())


def test_waits_begin_behind_the_kernels_in_front(s2d2):
    """A product that may be resident early, with waits of about 0.2 ms (a poll takes about 4 us), behind one that runs for more than a
    millisecond on half of the SMs: its own steps take microseconds, so that nothing runs out."""
    from paper_2603_25702_b200 import binding
    M, N, K = 37 * 256, 256, 1048576
    big = [(torch.randint(0, 256, (n * K // 2,), dtype=torch.uint8, device="cuda"),
            torch.full((s2d2.mxfp4_sizes(n, K)[1],), 100, dtype=torch.uint8, device="cuda")) for n in (M, N)]
    y = torch.empty(M, N, device="cuda")
    small = [((1, 4096, 256), 5), ((64, 384, 4096), 6), ((300, 6001, 320), 7)]
    for (m, n, k), seed in small:
        (x, xv), (w, wv) = operand(m, k, seed), operand(n, k, seed + 10, 0.02)
        z = torch.zeros(m, n, device="cuda")
        gemm(s2d2, big[0], big[1], y, M, N, K)
        binding.debug_mxfp4_wait(50)
        gemm(s2d2, x, w, z, m, n, k)
        s2d2.ops_status(stream())
        err = np.abs(z.double().cpu().numpy() - xv @ wv.T)
        assert (err <= product_tolerance(xv, wv, 1.0, "fp32")).all()


# a CTA per tile with one and with several tiles, clusters of two, four and eight that share k, pairs of CTAs with one and several tiles
@pytest.mark.parametrize("y_type", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(5, 37000, 256), (64, 8192, 2048), (1, 4096, 4096), (3, 130, 8192), (300, 6001, 320), (450, 30001, 300)])
def test_product_that_runs_out_is_nan_and_reported(s2d2, M, N, K, y_type):
    from paper_2603_25702_b200 import binding
    dt = {"fp32": torch.float32, "bf16": torch.bfloat16}[y_type]
    (x, xv), (w, _) = operand(M, K, 1), operand(N, K, 2, 0.02)
    pad = 3

    def call(y):
        s2d2.mxfp4_gemm(x[0].data_ptr(), x[1].data_ptr(), w[0].data_ptr(), w[1].data_ptr(), y.data_ptr(), y_type, M, N, K, N + pad,
                        stream=stream())

    want, y = (torch.full((M + 1, N + pad), 7.0, dtype=dt, device="cuda") for _ in range(2))
    call(want)
    s2d2.ops_status(stream())
    binding.debug_mxfp4_wait(64, True)
    call(y)
    with pytest.raises(s2d2.S2D2Error) as e:
        s2d2.ops_status(stream())
    assert e.value.code == -5
    assert y[:M, :N].isnan().all() and (y[:M, N:] == 7).all() and (y[M:] == 7).all()
    s2d2.ops_status(stream())                                        # reported once
    call(y)
    s2d2.ops_status(stream())
    assert torch.equal(y, want)                                      # and nothing of it is left


@pytest.mark.parametrize("M,N,K", [(8, 20000, 512), (100, 300, 64), (300, 20000, 128), (20000, 200, 32)])
def test_scores_that_run_out_are_nan_and_reported(s2d2, M, N, K):
    from paper_2603_25702_b200 import binding
    (x, _), (w, _) = operand(M, K, 1), operand(N, K, 2, 0.02)
    tok = torch.arange(M, dtype=torch.int32, device="cuda") % N
    ws = torch.zeros(s2d2.mxfp4_score_workspace(M, N, K), dtype=torch.uint8, device="cuda")

    def call():
        o = torch.full((3, M + 1), 7.0, device="cuda")
        s2d2.mxfp4_score(x[0].data_ptr(), x[1].data_ptr(), w[0].data_ptr(), w[1].data_ptr(), M, N, K, tok.data_ptr(), ws.data_ptr(),
                         ws.numel(), d_logprob=o[0].data_ptr(), d_lse=o[1].data_ptr(), d_entropy=o[2].data_ptr(), stream=stream())
        return o

    want = call()
    s2d2.ops_status(stream())
    binding.debug_mxfp4_wait(64, True)
    got = call()
    with pytest.raises(s2d2.S2D2Error) as e:
        s2d2.ops_status(stream())
    assert e.value.code == -5
    assert got[:, :M].isnan().all() and (got[:, M:] == 7).all()
    s2d2.ops_status(stream())
    assert torch.equal(call(), want)


def test_a_limit_that_is_not_reached_changes_nothing(s2d2):
    from paper_2603_25702_b200 import binding
    M, N, K = 64, 384, 4096
    (x, xv), (w, wv) = operand(M, K, 1), operand(N, K, 2, 0.02)
    a, b = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda")
    gemm(s2d2, x, w, a, M, N, K)
    binding.debug_mxfp4_wait(4096)
    gemm(s2d2, x, w, b, M, N, K)
    s2d2.ops_status(stream())
    assert torch.equal(a, b)
    for bad in (0, (1 << 20) + 1):
        with pytest.raises(s2d2.S2D2Error) as e:
            binding.debug_mxfp4_wait(bad)
        assert e.value.code == -1


def test_every_host_thread_learns_of_a_wait_that_ran_out(s2d2):
    """One thread's question does not take the answer from another, and nothing is left to be cleared on a stream."""
    import threading
    from paper_2603_25702_b200 import binding
    M, N, K = 5, 300, 256
    (x, xv), (w, wv) = operand(M, K, 1), operand(N, K, 2, 0.02)
    y = torch.zeros(M, N, device="cuda")
    torch.cuda.synchronize()
    launched, asked, codes = threading.Event(), threading.Event(), []

    def ask(raw):
        try:
            s2d2.ops_status(raw)
            return 0
        except s2d2.S2D2Error as e:
            return e.code

    def work():
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            ask(st.cuda_stream)                                      # a new thread is told of all earlier ones
            binding.debug_mxfp4_wait(64, True)
            gemm(s2d2, x, w, y, M, N, K)
            launched.set()
            asked.wait(60)
            codes.append(ask(st.cuda_stream))
            codes.append(ask(st.cuda_stream))
            gemm(s2d2, x, w, y, M, N, K)
            codes.append(ask(st.cuda_stream))

    t = threading.Thread(target=work)
    t.start()
    launched.wait(60)
    torch.cuda.synchronize()
    codes.append(ask(stream()))
    codes.append(ask(stream()))
    asked.set()
    t.join(60)
    assert codes == [-5, 0, -5, 0, 0], codes
    assert (np.abs(y.double().cpu().numpy() - xv @ wv.T) <= product_tolerance(xv, wv, 1.0, "fp32")).all()
