"""Rotary positions with norms (qk_rope) and the append to a paged cache (kv_append) against 64-bit restatements."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def stream():
    return torch.cuda.current_stream().cuda_stream


def near(got, want, size, dtype):
    tol = au.rope_tolerance(want, size, dtype)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


# rows, q heads, k heads, head_dim, rot_dim, row padding: whole vectors; a part of the head; an odd number of groups; elements one by one; nothing rotated
SHAPES = [(1, 32, 8, 128, 128, 0), (3, 5, 1, 64, 32, 64), (700, 3, 1, 80, 48, 16), (9, 2, 1, 96, 96, 3), (33, 1, 0, 66, 30, 1), (5, 0, 2, 7, 6, 0),
          (4, 3, 3, 128, 0, 0), (2, 1, 1, 512, 512, 0), (2500, 16, 4, 128, 64, 8), (40, 2, 2, 24, 24, 8), (17, 1, 1, 1, 0, 2)]


@pytest.mark.parametrize("rows,hq,hk,dim,rot,pad", SHAPES)
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [False, True])
def test_matches_the_definition(s2d2, rows, hq, hk, dim, rot, pad, dtype, layout, norm):
    g = torch.Generator(device="cuda").manual_seed(rows + dim)
    wide = (hq + hk) * dim + pad
    x = (torch.randn(rows, wide, generator=g, device="cuda") * 3).to(DT[dtype])
    q, k = x[:, :hq * dim].unflatten(1, (hq, dim)) if hq else x[:, :0], x[:, hq * dim:(hq + hk) * dim].unflatten(1, (hk, dim)) if hk else x[:, :0]
    pos = torch.randint(-5, 2000000, (rows,), generator=g, device="cuda", dtype=torch.int32)
    freqs = au.frequencies(rot).cuda()
    gains = [torch.rand(dim, generator=g, device="cuda") + 0.5 for _ in range(2)]
    qo, ko = (torch.full((rows, n * dim + 5), 7.0, dtype=DT[dtype], device="cuda") for n in (hq, hk))
    rope = s2d2.Rope(freqs.data_ptr() if rot else 0, rot, layout, 0.75, d_q_gain=gains[0].data_ptr() if norm else 0,
                     d_k_gain=gains[1].data_ptr() if norm else 0, eps=1e-3)
    s2d2.qk_rope(q.data_ptr(), qo.data_ptr(), hq, k.data_ptr(), ko.data_ptr(), hk, dtype, rows, dim, pos.data_ptr() if rot else 0, rope, q_stride=wide,
                 k_stride=wide, q_out_stride=qo.stride(0), k_out_stride=ko.stride(0), stream=stream())
    for n, a, b, gain in ((hq, q, qo, gains[0]), (hk, k, ko, gains[1])):
        if not n:
            continue
        want, size = au.rope(a, pos, freqs, rot, layout, 0.75, gain if norm else None, 1e-3)
        near(b[:, :n * dim].unflatten(1, (n, dim)), want, size, DT[dtype])
        assert (b[:, n * dim:] == 7).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dim,off", [(128, 0), (128, 1), (64, 8), (20, 0)])
def test_in_place_and_unaligned_buffers(s2d2, dtype, dim, off):
    rows, heads = 37, 6
    buf = torch.randn(rows * heads * dim + off, device="cuda").to(DT[dtype])
    x = buf[off:].view(rows, heads, dim)
    pos = torch.arange(rows, device="cuda", dtype=torch.int32)
    freqs = au.frequencies(dim).cuda()
    gain = torch.rand(dim, device="cuda") + 0.5
    want, size = au.rope(x, pos, freqs, dim, gain=gain)
    rope = s2d2.Rope(freqs.data_ptr(), dim, d_q_gain=gain.data_ptr())
    s2d2.qk_rope(x.data_ptr(), x.data_ptr(), heads, 0, 0, 0, dtype, rows, dim, pos.data_ptr(), rope, stream=stream())
    near(x, want, size, DT[dtype])


def test_far_positions_keep_their_angle(s2d2):
    """At position 2^31 - 1 the fastest pair has turned 3e8 times: in 32 bits its angle would be lost."""
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 123456789], device="cuda", dtype=torch.int32)
    freqs = au.frequencies(64).cuda()
    x = torch.randn(6, 2, 64, device="cuda")
    y = torch.empty_like(x)
    s2d2.qk_rope(x.data_ptr(), y.data_ptr(), 2, 0, 0, 0, "fp32", 6, 64, pos.data_ptr(), s2d2.Rope(freqs.data_ptr(), 64), stream=stream())
    near(y, *au.rope(x, pos, freqs, 64), torch.float32)
    assert torch.equal(y[0], x[0])


def test_special_values(s2d2):
    """A head of zeros stays zero; NaN and infinities stay in their head (with a norm) or in their pair."""
    x = torch.randn(4, 3, 64, device="cuda")
    x[0] = 0
    x[1, 1, 5] = float("nan")
    x[2, 2, 9] = float("inf")
    y = torch.empty_like(x)
    pos = torch.arange(4, device="cuda", dtype=torch.int32)
    freqs, gain = au.frequencies(64).cuda(), torch.ones(64, device="cuda")
    s2d2.qk_rope(x.data_ptr(), y.data_ptr(), 3, 0, 0, 0, "fp32", 4, 64, pos.data_ptr(), s2d2.Rope(freqs.data_ptr(), 64, d_q_gain=gain.data_ptr()), stream=stream())
    assert (y[0] == 0).all() and torch.isnan(y[1, 1]).all() and torch.isfinite(y[1, [0, 2]]).all()
    assert torch.isnan(y[2, 2, 9]) and torch.isfinite(y[2, :2]).all() and torch.isfinite(y[3]).all()
    s2d2.qk_rope(x.data_ptr(), y.data_ptr(), 3, 0, 0, 0, "fp32", 4, 64, pos.data_ptr(), s2d2.Rope(freqs.data_ptr(), 64), stream=stream())
    assert torch.isnan(y).nonzero().tolist() == [[1, 1, 5], [1, 1, 37]] and (~torch.isfinite(y[2])).sum() == 2


@pytest.mark.parametrize("lens", [[(1, 1)], [(8, 1031)], [(3, 3), (0, 5), (1, 64), (70, 200), (2, 1)], [(1, 65)] * 40, [(0, 0), (600, 1000)]])
@pytest.mark.parametrize("dim,hq,hkv,page,order,pad", [(128, 32, 8, 64, "head", 0), (64, 6, 2, 16, "token", 8), (80, 3, 1, 8, "head", 16), (72, 2, 2, 128, "token", 3),
                                                       (8, 0, 1, 8, "head", 0)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("norm,rotate", [(True, True), (False, True), (False, False)])
def test_append_matches_the_definition(s2d2, lens, dim, hq, hkv, page, order, pad, dtype, norm, rotate):
    b = au.Batch(lens, max(hq, hkv), hkv, dim, page, order, spare=3, poison=5.0)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, wide = b.n_rows, (hq + 2 * hkv) * dim + pad
    x = torch.randn(rows, wide, generator=g, device="cuda").to(DT[dtype])
    q, k, v = x[:, :hq * dim], x[:, hq * dim:(hq + hkv) * dim], x[:, (hq + hkv) * dim:(hq + 2 * hkv) * dim]
    gains = [torch.rand(dim, generator=g, device="cuda") + 0.5 for _ in range(2)]
    rot = dim if dim % 16 == 0 else dim // 2
    freqs = au.frequencies(rot).cuda()
    rope = s2d2.Rope(freqs.data_ptr(), rot, "interleaved", 1.25, d_q_gain=gains[0].data_ptr() if norm else 0,
                     d_k_gain=gains[1].data_ptr() if norm else 0) if rotate else None
    q_out = torch.full((rows, hq * dim + 1), 7.0, dtype=torch.bfloat16, device="cuda")
    before = b.cache.clone()
    s2d2.kv_append(k.data_ptr(), v.data_ptr(), dtype, b.rows(s2d2), b.kv(s2d2), rope, k_stride=wide, v_stride=wide, d_q=q.data_ptr(),
                   d_q_out=q_out.data_ptr(), n_q_heads=hq, q_stride=wide, q_out_stride=hq * dim + 1, stream=stream())
    want, size = before.double(), torch.zeros_like(before, dtype=torch.float64)
    view = lambda t, i: (t if order == "head" else t.transpose(2, 3))[:, i].transpose(1, 2)          # [page, token, head, dim]
    exact = torch.ones_like(before, dtype=torch.bool)
    for s, (n, kv) in enumerate(lens):
        at = slice(b.first[s], b.first[s] + n)
        j = torch.arange(kv - n, kv, device="cuda")
        turn = lambda t, heads, gain: au.rope(t[at].unflatten(1, (heads, dim)), j, freqs, rot, "interleaved", 1.25, gain if norm else None) if rotate \
            else (t[at].unflatten(1, (heads, dim)).double(),) * 2
        if hq and n:
            near(q_out[at, :hq * dim].unflatten(1, (hq, dim)), *turn(q, hq, gains[0]), torch.bfloat16)
        keep = j >= 0                                            # n > kv: the first rows have no place
        if not n or not bool(keep.any()):
            continue
        page_of, tok = b.table[s, j[keep] // page].long(), j[keep] % page
        yk, sk = turn(k, hkv, gains[1])
        view(want, 0)[page_of, tok], view(size, 0)[page_of, tok] = yk[keep], sk[keep]
        view(want, 1)[page_of, tok] = v[at].unflatten(1, (hkv, dim)).double()[keep]
        view(exact, 0)[page_of, tok] = view(exact, 1)[page_of, tok] = False
    assert torch.equal(b.cache[exact], before[exact])            # nothing else was touched
    near(b.cache, want, size, torch.bfloat16)
    assert (q_out[:, hq * dim:] == 7).all() and (q_out[b.first[-1]:] == 7).all()


def test_append_with_given_positions_and_without_queries(s2d2):
    """Verifier rows: the masked copies stand behind the drafted tokens in the cache but share their positions."""
    b = au.Batch([(16, 316), (16, 40)], 4, 2, 64)
    x = torch.randn(32, 4, 64, device="cuda")
    pos = torch.cat([torch.arange(300, 308).repeat(2), torch.arange(24, 32).repeat(2)]).int().cuda()
    freqs = au.frequencies(64).cuda()
    s2d2.kv_append(x.data_ptr(), x[:, 2:].data_ptr(), "fp32", b.rows(s2d2), b.kv(s2d2), s2d2.Rope(freqs.data_ptr(), 64), k_stride=256, v_stride=256,
                   d_pos=pos.data_ptr(), stream=stream())
    want, size = au.rope(x[:, :2], pos, freqs, 64)
    for s, (n, kv) in enumerate(b.lens):
        page, tok = (t[kv - n:] for t in b.places(s))
        near(b.k.transpose(1, 2)[page, tok], want[16 * s:16 * s + 16], size[16 * s:16 * s + 16], torch.bfloat16)
        assert torch.equal(b.v.transpose(1, 2)[page, tok], x[16 * s:16 * s + 16, 2:].bfloat16())


def test_append_follows_no_bad_length_page_or_row_list(s2d2):
    b = au.Batch([(2, 70), (2, 70), (2, 70), (2, 70)], 2, 1, 64, poison=5.0)
    before = b.cache.clone()
    x = torch.randn(8, 1, 64, device="cuda")
    b.table[0, 1] = b.n_pages                                    # a page that is not one
    b.table[1, 1] = -1
    b.kv_len[2] = b.max_pages * b.page + 1                       # more than the list holds
    b.kv_len[3] = -3
    s2d2.kv_append(x.data_ptr(), x.data_ptr(), "fp32", b.rows(s2d2), b.kv(s2d2), stream=stream())
    assert torch.equal(b.cache.view(torch.int16), before.view(torch.int16))
    for row0 in ([0, 9, 9, 9, 9], [-4, -2, 0, 0, 0], [0, 0, 0, 0, 0], [2 ** 31 - 1] * 5):
        b.row0.copy_(torch.tensor(row0, dtype=torch.int32))
        s2d2.kv_append(x.data_ptr(), x.data_ptr(), "fp32", b.rows(s2d2), b.kv(s2d2), stream=stream())
        assert torch.equal(b.cache.view(torch.int16), before.view(torch.int16)), row0


def test_append_beyond_32_bit_offsets(s2d2):
    """Pages 2^28 elements apart: the last one begins 5 GB behind the first."""
    stride, pages, dim = 1 << 28, 11, 64
    pool = torch.empty(stride * (pages - 1) + 2 * 64 * dim, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[10, 3]], dtype=torch.int32, device="cuda")
    row0, kv_len = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.tensor([66], dtype=torch.int32, device="cuda")
    x = torch.randn(3, 1, dim, device="cuda").bfloat16()
    kv = s2d2.PagedKV(pool.data_ptr(), pool[64 * dim:].data_ptr(), pages, 64, 1, dim, page_stride=stride, head_stride=64 * dim, token_stride=dim)
    s2d2.kv_append(x.data_ptr(), x.data_ptr(), "bf16", s2d2.Rows(3, 1, row0.data_ptr(), kv_len.data_ptr(), table.data_ptr(), 2), kv, stream=stream())
    assert torch.equal(pool[10 * stride + 63 * dim:][:dim], x[0, 0]) and torch.equal(pool[3 * stride:][:2 * dim].view(2, dim), x[1:, 0])
    assert torch.equal(pool[10 * stride + (64 + 63) * dim:][:dim], x[0, 0])
