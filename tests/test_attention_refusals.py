"""Argument checks of the attention-block operators that need no GPU, and the host-side frequencies."""
import math

import numpy as np
import pytest

P = 1 << 20     # a pointer value that no check may follow: every call below is refused before memory is looked at


@pytest.fixture(scope="module")
def s2d2():
    from paper_2603_25702_b200.build import build
    build()
    import paper_2603_25702_b200 as m
    return m


def refused(s2d2, text, fn, *a, code=-1, **kw):
    with pytest.raises(s2d2.S2D2Error) as e:
        fn(*a, **kw)
    assert e.value.code == code and text in str(e.value), str(e.value)


def kv(s2d2, n_pages=4, page=64, heads=2, dim=64, page_stride=None, head_stride=None, token_stride=None):
    t = dim if token_stride is None else token_stride
    h = t * page if head_stride is None else head_stride
    return s2d2.PagedKV(P, P, n_pages, page, heads, dim, page_stride=h * heads if page_stride is None else page_stride, head_stride=h, token_stride=t)


def rows(s2d2, n_rows=8, n_seqs=2, max_pages=3, max_rows=None):
    return s2d2.Rows(n_rows, n_seqs, P, P, P, max_pages, max_rows)


def test_frequencies(s2d2):
    f, scale = s2d2.rope_frequencies(128, 1e6)
    plain = 1e6 ** (-np.arange(64) / 64.0)
    assert scale == 1.0 and np.allclose(f, plain, rtol=1e-14, atol=0)
    f, scale = s2d2.rope_frequencies(128, 1e6, "linear", factor=4.0)
    assert scale == 1.0 and np.allclose(f, plain / 4, rtol=1e-14, atol=0)
    f, scale = s2d2.rope_frequencies(128, 1e6, "ntk", factor=4.0)
    assert f[0] == 1.0 and np.isclose(f[-1], plain[-1] / 4, rtol=1e-12)          # the slowest pair slows down by the whole factor
    f, scale = s2d2.rope_frequencies(128, 1e6, "yarn", factor=4.0, original_len=32768)
    turns = 32768 * plain / (2 * math.pi)
    assert np.isclose(scale, 0.1 * math.log(4) + 1, rtol=1e-6)
    assert np.allclose(f[turns > 40], plain[turns > 40]) and np.allclose(f[turns < 0.7], plain[turns < 0.7] / 4)
    assert (np.diff(f) < 0).all() and ((f <= plain * (1 + 1e-14)) & (f >= plain / 4 * (1 - 1e-14))).all()
    f, scale = s2d2.rope_frequencies(128, 1e6, "bands", factor=4.0, original_len=32768, turns_fast=4.0)
    keep = np.clip((turns - 1) / 3, 0, 1)
    assert scale == 1.0 and np.allclose(f, plain * keep + plain / 4 * (1 - keep), rtol=1e-12)
    f, _ = s2d2.rope_frequencies(2, 1e4)
    assert f.tolist() == [1.0]


def test_frequency_refusals(s2d2):
    f = s2d2.rope_frequencies
    for rot in (0, -2, 3, 514, 2 ** 32 + 2):
        refused(s2d2, "rot_dim", f, rot, 1e4)
    refused(s2d2, "base", f, 64, 1.0)
    refused(s2d2, "base", f, 64, math.nan)
    refused(s2d2, "scaling", f, 64, 1e4, "other")
    refused(s2d2, "factor", f, 64, 1e4, "linear", factor=0.5)
    refused(s2d2, "factor", f, 64, 1e4, "ntk", factor=math.inf)
    refused(s2d2, "ntk", f, 2, 1e4, "ntk", factor=2.0)
    refused(s2d2, "original_len", f, 64, 1e4, "yarn", factor=2.0)
    refused(s2d2, "turns_fast", f, 64, 1e4, "yarn", factor=2.0, original_len=100, turns_fast=1.0)
    refused(s2d2, "turns_fast", f, 64, 1e4, "bands", factor=2.0, original_len=100, turns_slow=0.0)


def test_rope_refusals(s2d2):
    def call(dtype="fp32", rows=4, dim=64, hq=2, hk=1, rope=None, **kw):
        s2d2.qk_rope(P, P, hq, P, P, hk, dtype, rows, dim, P, rope or s2d2.Rope(P, 64), **kw)
    refused(s2d2, "layout", s2d2.Rope, P, 64, "other")
    refused(s2d2, "dtype", call, "fp16")
    refused(s2d2, "n_rows", call, rows=-1)
    refused(s2d2, "n_rows", call, rows=2 ** 31 + 1)
    refused(s2d2, "n_rows", call, rows=2 ** 64 + 1)
    refused(s2d2, "n_q_heads", call, hq=-1)
    refused(s2d2, "n_q_heads", call, hq=4097)
    refused(s2d2, "n_k_heads", call, hk=2 ** 32 + 1)
    refused(s2d2, "head_dim", call, dim=0)
    refused(s2d2, "head_dim", call, dim=513)
    refused(s2d2, "rot_dim", call, dim=62)
    refused(s2d2, "rot_dim", call, rope=s2d2.Rope(P, 63))
    refused(s2d2, "rot_dim", call, rope=s2d2.Rope(P, -2))
    refused(s2d2, "scale", call, rope=s2d2.Rope(P, 64, scale=math.inf))
    refused(s2d2, "eps", call, rope=s2d2.Rope(P, 64, eps=-1.0))
    refused(s2d2, "eps", call, rope=s2d2.Rope(P, 64, eps=math.nan))
    refused(s2d2, "q_stride", call, q_stride=127)
    refused(s2d2, "q_out_stride", call, q_out_stride=127)
    refused(s2d2, "k_stride", call, k_stride=2 ** 41)
    refused(s2d2, "k_out_stride", call, k_out_stride=0)


def test_append_refusals(s2d2):
    def call(dtype="fp32", r=None, c=None, rope=None, **kw):
        s2d2.kv_append(P, P, dtype, r or rows(s2d2), c or kv(s2d2), rope, **kw)
    refused(s2d2, "dtype", call, "int8")
    refused(s2d2, "n_rows", call, r=rows(s2d2, -1, max_rows=1))
    refused(s2d2, "n_seqs", call, r=rows(s2d2, n_seqs=-1))
    refused(s2d2, "max_pages", call, r=rows(s2d2, max_pages=2 ** 32))
    refused(s2d2, "max_rows", call, r=rows(s2d2, max_rows=0))
    refused(s2d2, "max_rows", call, r=rows(s2d2, max_rows=9))
    refused(s2d2, "n_pages", call, c=kv(s2d2, n_pages=0))
    for page in (0, 4, 24, 2 ** 21):
        refused(s2d2, "page_tokens", call, c=kv(s2d2, page=page))
    refused(s2d2, "n_kv_heads", call, c=kv(s2d2, heads=0))
    for dim in (0, 4, 60, 520):
        refused(s2d2, "head_dim", call, c=kv(s2d2, dim=dim))
    refused(s2d2, "strides", call, c=kv(s2d2, token_stride=68))
    refused(s2d2, "strides", call, c=kv(s2d2, page_stride=-64 * 128))
    refused(s2d2, "strides", call, c=kv(s2d2, page_stride=2 ** 39))
    refused(s2d2, "overlap", call, c=kv(s2d2, token_stride=56))
    refused(s2d2, "overlap", call, c=kv(s2d2, head_stride=64 * 64 - 8, page_stride=2 * 64 * 64))
    refused(s2d2, "overlap", call, c=kv(s2d2, page_stride=64 * 64))
    refused(s2d2, "overlap", call, c=kv(s2d2, token_stride=64, head_stride=64, page_stride=64 * 128))
    refused(s2d2, "rot_dim", call, rope=s2d2.Rope(P, 128))
    refused(s2d2, "k_stride", call, k_stride=127)
    refused(s2d2, "v_stride", call, v_stride=127)
    refused(s2d2, "q_stride", call, d_q=P, n_q_heads=2, q_stride=1)
    refused(s2d2, "q_out_stride", call, d_q=P, n_q_heads=2, q_out_stride=1)
    refused(s2d2, "n_q_heads", call, d_q=P, n_q_heads=-1)


def test_attention_refusals(s2d2):
    def call(heads=4, r=None, c=None, ws=1 << 40, **kw):
        s2d2.paged_attention(P, P, heads, r or rows(s2d2), c or kv(s2d2), P, ws, **kw)
    need = s2d2.paged_attention_workspace(rows(s2d2), kv(s2d2), 4)
    assert need >= 0 and need % 16 == 0
    refused(s2d2, "n_q_heads", call, heads=3)
    refused(s2d2, "n_q_heads", call, heads=0)
    refused(s2d2, "n_q_heads", s2d2.paged_attention_workspace, rows(s2d2), kv(s2d2), 5)
    refused(s2d2, "head_dim", call, c=kv(s2d2, dim=136), code=-6)
    refused(s2d2, "max_rows", call, r=rows(s2d2, max_rows=-1))
    refused(s2d2, "q_stride", call, q_stride=255)
    refused(s2d2, "q_stride", call, q_stride=260)
    refused(s2d2, "out_stride", call, out_stride=8)
    refused(s2d2, "mask_block", call, mask_block=-1)
    refused(s2d2, "mask_block", call, mask_block=2 ** 32 + 1)
    refused(s2d2, "mask_block", call, mask_block=1, d_row_mask=P)
    for scale in (0.0, -1.0, math.nan, math.inf):
        refused(s2d2, "scale", call, scale=scale)


def test_attention_limits(s2d2):
    """Sizes whose indices or counts would not fit are refused before any memory is looked at, and so is a workspace that is too small."""
    def both(heads, r, c, text):
        refused(s2d2, text, s2d2.paged_attention_workspace, r, c, heads, code=-6)
        refused(s2d2, text, s2d2.paged_attention, P, P, heads, r, c, P, 1 << 40, code=-6)
    both(4, rows(s2d2, n_rows=(1 << 22) + 1), kv(s2d2), "n_rows must be at most 2^22")
    both(4, rows(s2d2, max_pages=1 << 25), kv(s2d2), "max_pages * page_tokens")
    both(4, rows(s2d2, max_pages=2 ** 31 - 1), kv(s2d2, page=1 << 20), "max_pages * page_tokens")
    both(4096, rows(s2d2, n_rows=1 << 22), kv(s2d2, heads=1), "n_rows * n_q_heads / n_kv_heads")
    refused(s2d2, "too much", s2d2.paged_attention, P, P, 64, rows(s2d2, n_rows=1 << 20, max_pages=1 << 20), kv(s2d2, heads=64), P, 1 << 40, code=-6)
    for heads, r, c in ((4, rows(s2d2), kv(s2d2)), (64, rows(s2d2, n_rows=5000), kv(s2d2, heads=8, dim=128))):
        need = s2d2.paged_attention_workspace(r, c, heads)
        assert 0 < need <= 148 * (32 + 2 * 256 * (8 + 128 * 4))
        for ws in (need - 1, 0, -1):
            refused(s2d2, "workspace", s2d2.paged_attention, P, P, heads, r, c, P, ws)


def test_attention_strides_that_no_copy_can_have(s2d2):
    for q in (1 << 39, 1 << 40, -8):
        refused(s2d2, "q_stride", s2d2.paged_attention, P, P, 4, rows(s2d2), kv(s2d2), P, 1 << 40, q_stride=q)
    refused(s2d2, "out_stride", s2d2.paged_attention, P, P, 4, rows(s2d2), kv(s2d2), P, 1 << 40, out_stride=(1 << 40) + 8)


def test_attention_wait_tap(s2d2):
    from paper_2603_25702_b200 import binding
    for bad in (0, (1 << 20) + 1):
        refused(s2d2, "limit_polls", binding.debug_attention_wait, bad)
