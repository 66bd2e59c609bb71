"""MXFP4 conversions of matrices large enough for several steps per warp: every code, scale byte and value, bit for bit."""
import numpy as np
import pytest

from tests import ops_util as ou
from tests.test_gpu_mxfp4 import DT, quantize, stream

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
# whole groups of 1024 columns; a vector body with a tail; odd strides and first elements; a width between the groups; a multiple
# of 256; a short matrix of many columns; many short rows
@pytest.mark.parametrize("rows,cols,pad,lead", [(9473, 1024, 0, 0), (9500, 1056, 8, 0), (9473, 1001, 2, 3), (1000, 9728, 0, 0),
                                                (9500, 768, 0, 8), (129, 40000, 0, 0), (150000, 5, 0, 1), (9473, 257, 7, 0)])
def test_large_conversions(s2d2, dtype, rows, cols, pad, lead):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    buf = torch.randn(rows * (cols + pad) + lead, generator=g, device="cuda")
    buf *= torch.exp(3 * torch.randn(buf.shape, generator=g, device="cuda"))
    at = torch.randint(0, buf.numel(), (60,), generator=g, device="cuda")
    buf[at] = torch.tensor([float("nan"), float("inf"), -float("inf"), 0.0, 1e-40, 3e38], device="cuda").repeat(10)
    x = buf.to(DT[dtype])[lead:].view(rows, cols + pad)[:, :cols]
    codes, scales = quantize(s2d2, x)
    outs = {}
    for out in DT:
        outs[out] = y = torch.full((rows * (cols + pad) + lead + 16,), 7.0, dtype=DT[out], device="cuda")
        s2d2.mxfp4_dequantize(codes.data_ptr(), scales.data_ptr(), rows, cols, y[lead:].data_ptr(), out, cols + pad, stream())
        assert (y[:lead] == 7).all() and (y[lead + rows * (cols + pad):] == 7).all()
        outs[out] = y[lead:lead + rows * (cols + pad)].view(rows, cols + pad)
        assert (outs[out][:, cols:] == 7).all()
    nb = ou.n_blocks(cols)
    all_scales = np.zeros((rows, nb), np.uint8)
    got_codes = codes[:-64].view(rows, nb * 16).cpu().numpy()
    step = max(1, 2 ** 20 // cols)
    for r in range(0, rows, step):                                   # the oracle in parts: its intermediates are large
        part = x[r:r + step].double().cpu().numpy()
        c, s = ou.mxfp4_encode(part)
        all_scales[r:r + step] = s
        assert np.array_equal(got_codes[r:r + step], c), r
        want = ou.mxfp4_values(c, s, cols)
        for out in DT:
            got = outs[out][r:r + step, :cols].double().cpu().numpy()
            with np.errstate(over="ignore"):
                limit = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
            assert np.array_equal(got, limit, equal_nan=True), (r, out)
    want_s = ou.tile_scales(all_scales)
    got_s = scales.cpu().numpy()
    assert np.array_equal(got_s[:want_s.size], want_s)
    assert (got_s[want_s.size:] == 0xA5).all() and (codes[-64:] == 0xA5).all()
