"""Argument checks of the stand-alone operators that need no GPU, and pins of the 64-bit restatements the GPU tests use."""
import numpy as np
import pytest

from tests import ops_util as ou

P = 1 << 20     # a pointer value that no check may follow: every call below is refused before memory is looked at


@pytest.fixture(scope="module")
def s2d2():
    from paper_2603_25702_b200.build import build
    build()
    import paper_2603_25702_b200 as m
    return m


def refused(s2d2, code, text, fn, *a, **kw):
    with pytest.raises(s2d2.S2D2Error) as e:
        fn(*a, **kw)
    assert e.value.code == code and text in str(e.value), str(e.value)


def test_sizes(s2d2):
    assert s2d2.mxfp4_sizes(1, 1) == (16, 512)
    assert s2d2.mxfp4_sizes(128, 128) == (128 * 64, 512)
    assert s2d2.mxfp4_sizes(129, 129) == (129 * 80, 4 * 512)
    assert s2d2.mxfp4_sizes(0, 32) == (0, 0)
    assert s2d2.mxfp4_sizes(151936, 4096) == (151936 * 2048, 1187 * 32 * 512)
    refused(s2d2, -1, "rows", s2d2.mxfp4_sizes, -1, 32)
    refused(s2d2, -1, "columns", s2d2.mxfp4_sizes, 1, 0)


def test_sizes_agree_with_the_library(s2d2):
    """The binding computes sizes inside the limits itself; the library's entry point gives the same, and the refusals."""
    import ctypes as C
    from paper_2603_25702_b200.binding import load_library
    lib = load_library()
    rng = np.random.default_rng(0)
    shapes = [(0, 1), (4194304, 1048576)] + [(int(r), int(c)) for r, c in np.exp(rng.uniform(0, 13, (200, 2)))]
    for rows, cols in shapes:
        a, b = C.c_int64(), C.c_int64()
        assert lib.s2d2_mxfp4_sizes(rows, cols, C.byref(a), C.byref(b)) == 0
        assert s2d2.mxfp4_sizes(rows, cols) == (a.value, b.value), (rows, cols)
    refused(s2d2, -1, "rows", s2d2.mxfp4_sizes, 4194305, 1)
    refused(s2d2, -1, "columns", s2d2.mxfp4_sizes, 1, 1048577)


def test_quantize_refusals(s2d2):
    q, d = s2d2.mxfp4_quantize, s2d2.mxfp4_dequantize
    refused(s2d2, -1, "dtype", q, P, "fp16", 1, 32, 32, P, P)
    refused(s2d2, -1, "rows", q, P, "fp32", -1, 32, 32, P, P)
    refused(s2d2, -1, "columns", q, P, "fp32", 1, 0, 32, P, P)
    refused(s2d2, -1, "row_stride", q, P, "fp32", 1, 32, 31, P, P)
    refused(s2d2, -1, "row_stride", d, P, P, 1, 32, P, "bf16", 31)
    refused(s2d2, -1, "rows", d, P, P, (1 << 22) + 1, 32, P, "bf16", 32)


def test_product_refusals(s2d2):
    g = s2d2.mxfp4_gemm
    refused(s2d2, -1, "dtype", g, P, P, P, P, P, "int8", 1, 1, 32)
    refused(s2d2, -1, "M must", g, P, P, P, P, P, "fp32", -1, 1, 32)
    refused(s2d2, -1, "N must", g, P, P, P, P, P, "fp32", 1, 0, 32)
    refused(s2d2, -1, "K must", g, P, P, P, P, P, "fp32", 1, 1, 0)
    refused(s2d2, -1, "K must", g, P, P, P, P, P, "fp32", 1, 1, (1 << 20) + 1)
    refused(s2d2, -1, "y_stride", g, P, P, P, P, P, "fp32", 2, 8, 32, 7)


def test_score_refusals(s2d2):
    f = s2d2.score_logits
    refused(s2d2, -1, "dtype", f, P, "fp64", 1, 8, 8, d_lse=P)
    refused(s2d2, -1, "n_rows", f, P, "fp32", -1, 8, 8, d_lse=P)
    refused(s2d2, -1, "vocab", f, P, "fp32", 1, 0, 8, d_lse=P)
    refused(s2d2, -1, "vocab", f, P, "fp32", 1, (1 << 21) + 1, 1 << 22, d_lse=P)
    refused(s2d2, -1, "row_stride", f, P, "fp32", 1, 8, 7, d_lse=P)
    refused(s2d2, -1, "row_stride", f, P, "fp32", 1 << 40, 8, 1 << 40, d_lse=P)
    refused(s2d2, -1, "top_k", f, P, "fp32", 1, 8, 8, P, 33, d_top_ids=P)
    refused(s2d2, -1, "top_k", f, P, "fp32", 1, 8, 8, P, -1, d_top_ids=P)
    refused(s2d2, -1, "tokens", f, P, "fp32", 1, 8, 8, d_logprob=P)
    refused(s2d2, -1, "tokens", f, P, "fp32", 1, 8, 8, d_rank=P)
    refused(s2d2, -1, "top_k", f, P, "fp32", 1, 8, 8, P, 4, d_lse=P)
    refused(s2d2, -1, "top_k", f, P, "fp32", 1, 8, 8, P, 0, d_top_ids=P)
    refused(s2d2, -1, "no output", f, P, "fp32", 1, 8, 8, P)


def test_sizes_beyond_32_bits_are_not_cut_off(s2d2):
    big = 2 ** 32 + 4
    refused(s2d2, -1, "M must", s2d2.mxfp4_gemm, P, P, P, P, P, "fp32", big, 1, 32, 1)
    refused(s2d2, -1, "N must", s2d2.mxfp4_gemm, P, P, P, P, P, "fp32", 1, big, 32, big)
    refused(s2d2, -1, "K must", s2d2.mxfp4_gemm, P, P, P, P, P, "fp32", 1, 1, big, 1)
    refused(s2d2, -1, "vocab", s2d2.score_logits, P, "fp32", 1, big, big, d_lse=P)
    refused(s2d2, -1, "top_k", s2d2.score_logits, P, "fp32", 1, 8, 8, P, big, d_top_ids=P)
    refused(s2d2, -1, "M must", s2d2.mxfp4_score_workspace, big, 100, 32)
    refused(s2d2, -1, "M must", s2d2.mxfp4_score, P, P, P, P, big, 100, 32, P, P, 1 << 30, d_lse=P)


def test_hidden_score_refusals(s2d2):
    f, need = s2d2.mxfp4_score, s2d2.mxfp4_score_workspace(4, 1000, 64)
    assert need > 0 and need % 16 == 0 and s2d2.mxfp4_score_workspace(0, 1000, 64) == 0
    refused(s2d2, -1, "N must", s2d2.mxfp4_score_workspace, 1, 0, 32)
    refused(s2d2, -1, "M must", f, P, P, P, P, -1, 1000, 64, P, P, need, d_lse=P)
    refused(s2d2, -1, "no output", f, P, P, P, P, 4, 1000, 64, P, P, need)
    refused(s2d2, -1, "tokens", f, P, P, P, P, 4, 1000, 64, 0, P, need, d_logprob=P)
    refused(s2d2, -1, "workspace", f, P, P, P, P, 4, 1000, 64, P, P, need - 1, d_lse=P)


def test_no_gpu_fails_loudly(s2d2):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(s2d2.S2D2Error) as e:
        s2d2.score_logits(P, "fp32", 1, 8, 8, d_lse=P)
    assert e.value.code == -2


def test_restated_quantisation_on_known_blocks():
    x = np.zeros((1, 32))
    x[0, :8] = [6, -6, 5, 3.5, 2.5, 1.75, 0.25, -0.75]               # scale 1: ties go to the even code
    codes, scales = ou.mxfp4_encode(x)
    assert scales.tolist() == [[127]]
    assert ou.mxfp4_values(codes, scales, 8).tolist() == [[6, -6, 4, 4, 2, 2, 0, -1]]
    x[0, 0] = 7.99                                                   # floor(log2 7.99) is 2: above 6 saturates
    codes, scales = ou.mxfp4_encode(x)
    assert scales.tolist() == [[127]] and ou.mxfp4_values(codes, scales, 1).tolist() == [[6]]
    codes, scales = ou.mxfp4_encode(np.full((1, 3), 2.0 ** -149))
    assert scales.tolist() == [[0]] and ou.mxfp4_values(codes, scales, 3).tolist() == [[0, 0, 0]]
    _, scales = ou.mxfp4_encode(np.array([[1.0, np.inf], [1.0, np.nan], [0.0, 0.0]]))
    assert scales.tolist() == [[255], [255], [0]]


def test_restated_values_are_nearest():
    """No e2m1 value times the block's scale lies nearer to an element than the chosen one (magnitudes up to 6 scales)."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((20, 96)) * np.exp(rng.standard_normal((20, 1)) * 3)
    codes, scales = ou.mxfp4_encode(x)
    v = ou.mxfp4_values(codes, scales, 96)
    unit = np.repeat(np.exp2(scales.astype(float) - 127), 32, axis=1)
    all_values = np.concatenate([-ou.GRID, ou.GRID])
    best = np.abs(x[:, :, None] - all_values * unit[:, :, None]).min(axis=2)
    assert (np.abs(x - v) == best).all()


def test_restated_scores_on_a_closed_form():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125]]))
    o = ou.scores(x, [2], 3)
    assert np.allclose(o["logprob"], np.log(0.125)) and o["rank"].tolist() == [2] and np.allclose(o["lse"], 0)
    assert np.allclose(o["entropy"], 1.75 * np.log(2)) and o["top_ids"].tolist() == [[0, 1, 2]]
