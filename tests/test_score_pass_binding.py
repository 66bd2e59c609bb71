"""What Engine.score_pass and the operators' functions hand to the library: nothing is cut off to 32 or 64 bits (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

from tests.test_ops_refusals import P, refused, s2d2  # noqa: F401


class Recorder:
    """Stands in for the library: keeps the arguments of s2d2_score_pass, and the tokens they point to."""

    def __init__(self, rc=0):
        self.rc, self.calls, self.tokens = rc, [], None

    def s2d2_score_pass(self, h, which, n_rows, tokens, top_k, *outs):
        self.calls.append((which, n_rows, top_k, [o is not None for o in outs]))
        if tokens:
            self.tokens = list((C.c_int32 * n_rows).from_address(tokens))
        return self.rc

    def s2d2_last_error(self, h):
        return b"refused"


def engine(s2d2, rc=0):  # noqa: F811
    e = object.__new__(s2d2.Engine)
    e.lib, e._h = Recorder(rc), None
    return e


@pytest.mark.parametrize("tokens", [[5, -1, 2 ** 32 + 5, 2 ** 31], np.array([5, -7, 2 ** 32 + 5, -(2 ** 32) + 3]),
                                    np.array([5, 2 ** 64 - 1, 2 ** 32, 2 ** 31], dtype=np.uint64)])
def test_tokens_beyond_32_bits_stay_outside_the_vocabulary(s2d2, tokens):  # noqa: F811
    e = engine(s2d2)
    out = e.score_pass(0, 4, tokens)
    assert e.lib.tokens == [5, -1, -1, -1]
    assert set(out) == {"lse", "entropy", "logprob", "rank"}


@pytest.mark.parametrize("top_k", [2 ** 32 + 4, -1, 33, 2 ** 62])
def test_a_top_k_beyond_the_limit_reaches_the_library_as_one(s2d2, top_k):  # noqa: F811
    e = engine(s2d2, rc=-1)
    with pytest.raises(s2d2.S2D2Error):
        e.score_pass(0, 2, None, top_k)
    (_, _, k, given), = e.lib.calls
    assert not 0 <= k <= 32 and not any(given[4:])


@pytest.mark.parametrize("n_rows", [-1, 2 ** 32 + 1, -(2 ** 40)])
def test_row_counts_outside_of_32_bits_are_refused_by_the_library(s2d2, n_rows):  # noqa: F811
    e = engine(s2d2, rc=-1)
    with pytest.raises(s2d2.S2D2Error):
        e.score_pass(0, n_rows, None, 5)
    assert e.lib.calls[0][1] == -1 or e.lib.calls[0][1] == n_rows < 0


def test_sizes_beyond_64_bits_are_not_cut_off(s2d2):  # noqa: F811
    big = 2 ** 64
    refused(s2d2, -1, "rows", s2d2.mxfp4_sizes, big + 1, 32)
    refused(s2d2, -1, "columns", s2d2.mxfp4_sizes, 1, big + 32)
    refused(s2d2, -1, "rows", s2d2.mxfp4_quantize, P, "fp32", big, 32, 32, P, P)
    refused(s2d2, -1, "columns", s2d2.mxfp4_quantize, P, "fp32", 1, big + 32, 32, P, P)
    refused(s2d2, -1, "row_stride", s2d2.mxfp4_quantize, P, "fp32", 1, 32, big + 32, P, P)
    refused(s2d2, -1, "row_stride", s2d2.mxfp4_dequantize, P, P, 1, 32, P, "fp32", big + 32)
    refused(s2d2, -1, "y_stride", s2d2.mxfp4_gemm, P, P, P, P, P, "fp32", 1, 8, 32, big + 8)
    refused(s2d2, -1, "n_rows", s2d2.score_logits, P, "fp32", big, 8, 8, d_lse=P)
    refused(s2d2, -1, "row_stride", s2d2.score_logits, P, "fp32", 1, 8, big + 8, d_lse=P)
    refused(s2d2, -1, "workspace", s2d2.mxfp4_score, P, P, P, P, 4, 1000, 64, P, P, big + 2 ** 40, d_lse=P)
