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
