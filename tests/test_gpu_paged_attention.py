"""Attention of new rows over a paged cache against a 64-bit restatement."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def run(s2d2, lens, heads=8, kv_heads=2, dim=128, mask_block=1, row_mask=None, scale=None, **kw):
    b = au.Batch(lens, heads, kv_heads, dim, **kw)
    got = b.attend(s2d2, mask_block, row_mask, scale)
    b.check(got, b.want(mask_block, row_mask, scale))
    s2d2.ops_status(torch.cuda.current_stream().cuda_stream)
    return b, got


# one token; lengths around the tiles; nothing cached; fewer cached than new; slots with nothing to do; a page that ends inside a tile
LENS = [[(1, 1)], [(1, 127), (1, 128), (1, 129), (1, 255), (1, 256), (1, 257)], [(5, 5)], [(130, 130)], [(0, 9), (1, 700), (0, 0), (3, 2), (2, 0), (1, 63)],
        [(64, 1000)], [(257, 300), (1, 2000), (33, 33)], [(1, 5000)], [(300, 3001)]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("mask_block", [1, 0, 32])
def test_lengths_and_masks(s2d2, lens, dim, mask_block):
    run(s2d2, lens, dim=dim, mask_block=mask_block, spare=2)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (3, 1), (10, 2), (32, 8), (24, 3), (71, 1), (160, 1)])
@pytest.mark.parametrize("lens", [[(1, 300)], [(40, 170), (2, 90)]])
def test_groups_of_heads(s2d2, heads, kv_heads, lens):
    run(s2d2, lens, heads, kv_heads, 64)


@pytest.mark.parametrize("dim", [8, 24, 32, 40, 64, 72, 80, 96, 120, 128])
@pytest.mark.parametrize("order", ["head", "token"])
def test_head_sizes_and_orders(s2d2, dim, order):
    run(s2d2, [(1, 200), (70, 260)], 4, 2, dim, order=order, q_pad=8, gap=8)


@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256, 4096])
@pytest.mark.parametrize("order", ["head", "token"])
def test_pages(s2d2, page, order):
    run(s2d2, [(1, 1), (1, 517), (20, 300), (150, 150)], 4, 2, 128, page=page, order=order)


@pytest.mark.parametrize("mask_block", [2, 3, 8, 100, 2 ** 31 - 1])
def test_blocks(s2d2, mask_block):
    run(s2d2, [(7, 7), (16, 500), (1, 9), (200, 201), (5, 3)], mask_block=mask_block, dim=64)


@pytest.mark.parametrize("lens", [[(16, 16)], [(16, 1040), (8, 200), (2, 2)], [(64, 64), (33, 700), (1, 1), (0, 4)], [(64, 2000)]])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (4, 4, 64), (5, 1, 80)])
def test_verifier_rows(s2d2, lens, heads, kv_heads, dim):
    run(s2d2, lens, heads, kv_heads, dim, 0, au.verifier_masks(lens, 1), spare=1)


def test_row_masks_of_any_bits(s2d2):
    """Rows that see nothing, single bits, bits of rows that do not exist, more rows than bits, nothing cached in front."""
    lens = [(40, 40), (3, 130), (70, 100), (64, 64), (2, 1)]
    g = torch.Generator().manual_seed(3)
    bits = torch.randint(-2 ** 63, 2 ** 63 - 1, (179,), generator=g, dtype=torch.int64)
    bits[:10] = 0
    bits[10] = 1 << 39
    bits[11] = 1 << 50
    bits[12] = -1
    _, (out, lse) = run(s2d2, lens, 4, 2, 128, 0, bits.cuda())
    assert (out[:10] == 0).all() and torch.isneginf(lse[:10]).all() and (out[11] == 0).all()


@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_scales(s2d2, scale):
    """Up to one key that takes everything, with a maximum that rises from tile to tile."""
    b = au.Batch([(20, 900), (1, 2000)], 4, 2, 64)
    for s, (_, kv) in enumerate(b.lens):
        b.keys[s].mul_(torch.linspace(0.1, 2, kv, device="cuda").bfloat16()[:, None, None])
    b.write()
    b.check(b.attend(s2d2, scale=scale), b.want(scale=scale))


@pytest.mark.parametrize("lens", [[(1, 400)], [(30, 260)], [(200, 400)]])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -1e30])
def test_what_a_row_does_not_see_has_no_influence(s2d2, lens, value):
    """Rubbish in keys and values of later tokens of the chunk: rows in front of it do not see it, rows behind it do."""
    b = au.Batch(lens, 4, 2, 128)
    n, kv = lens[0]
    at = kv - n + n // 2
    if n > 1:
        b.keys[0][at, 0] = value
        b.values[0][at, 1] = value
        b.values[0][at + 1, 1, 3] = value
    b.write()
    want = b.want()
    got = b.attend(s2d2)
    b.check(got, want)
    if n > 1:
        assert torch.isfinite(got[0][:n // 2]).all() and torch.isfinite(got[1][:n // 2]).all()


def test_masked_rows_with_nan_among_the_rows_they_do_not_see(s2d2):
    lens = [(16, 200), (64, 64)]
    mask = au.verifier_masks(lens)
    b = au.Batch(lens, 4, 2, 128)
    b.values[0][200 - 3] = float("nan")       # a masked copy: only it sees itself
    b.keys[1][63] = float("inf")
    b.write()
    got = b.attend(s2d2, 0, mask)
    b.check(got, b.want(0, mask))
    assert torch.isfinite(got[0][:13]).all() and torch.isnan(got[0][13]).all() and torch.isfinite(got[0][14:16 + 63]).all()


def test_infinite_and_nan_queries_stay_in_their_row(s2d2):
    b = au.Batch([(6, 300), (1, 50)], 4, 2, 64)
    b.q[2, 1] = float("inf")
    b.q[4, 3, 7] = float("nan")
    out, lse = b.attend(s2d2)
    hit = torch.zeros(7, 4, dtype=torch.bool, device="cuda")
    hit[2, 1] = hit[4, 3] = True
    assert torch.isnan(out).all(2).equal(hit) and torch.isnan(out).any(2).equal(hit) and torch.isnan(lse).equal(hit)


def test_bad_lengths_pages_and_row_lists_are_not_followed(s2d2):
    b = au.Batch([(2, 200), (2, 200), (2, 200), (2, 200), (2, 200)], 4, 2, 64, spare=1)
    want = b.want()
    b.table[0, 1] = b.n_pages
    b.table[1, 0] = -1
    b.kv_len[2] = b.max_pages * b.page + 1
    b.kv_len[3] = -3
    got = b.attend(s2d2)
    assert torch.isnan(got[0][:8]).all() and torch.isnan(got[1][:8]).all()
    for g, w, t in zip(got, want[:2], want[2:]):
        assert ((g[8:].double() - w[8:]).abs() <= t[8:]).all()
    for row0 in ([0, 12, 12, 12, 12, 12], [-4, -2, 0, 0, 0, 0], [0] * 6, [2 ** 31 - 1] * 6, [11, 11, 11, 11, 11, 5]):
        b.row0.copy_(torch.tensor(row0, dtype=torch.int32))
        out, lse = b.attend(s2d2)
        assert (out == 7).all() and (lse == 7).all(), row0


def test_offsets_beyond_32_bits(s2d2):
    """Pages 2^28 elements apart: the last one begins 5 GB behind the first."""
    b = au.Batch([(3, 300), (1, 130)], 4, 2, 128, n_spare_pages=1)
    want = b.want()
    stride = 1 << 28
    one = 2 * 2 * 64 * 128
    pool = torch.empty(stride * (b.n_pages - 1) + one, dtype=torch.bfloat16, device="cuda")
    for i in range(b.n_pages):
        pool[i * stride:i * stride + one] = b.cache[i].flatten()
    k = torch.as_strided(pool, (b.n_pages, 2, 64, 128), (stride, 64 * 128, 128, 1))
    b.k, b.v = k, torch.as_strided(pool, k.shape, k.stride(), storage_offset=2 * 64 * 128)
    b.check(b.attend(s2d2), want)


def test_host_bound_on_rows_does_not_change_results_beyond_rounding(s2d2):
    b = au.Batch([(1, 700), (90, 400), (3, 3)], 8, 2, 128)
    want = b.want()
    for max_rows in (1, 16, 90, 94):
        b.check(b.attend(s2d2, max_rows=max_rows), want)


def test_many_sequences(s2d2):
    g = torch.Generator().manual_seed(5)
    lens = [(int(n), int(n + c)) for n, c in zip(torch.randint(0, 4, (1500,), generator=g), torch.randint(0, 90, (1500,), generator=g))]
    run(s2d2, lens, 2, 1, 64, page=16)


@pytest.mark.parametrize("n", [1, 40, 300])
def test_many_units_per_cta(s2d2, n):
    """Items far longer than the ring of tiles, short ones in front of and behind them."""
    run(s2d2, [(1, 60), (n, 30000), (n, 31000), (0, 100), (n, 300), (2, 29000), (1, 5)], 4, 4, 64, seed=n)


def test_without_lse_and_with_output_padding(s2d2):
    b = au.Batch([(4, 90), (130, 200)], 4, 2, 64)
    want = b.want()
    b.check(b.attend(s2d2, lse=False, out_pad=16), want)


def test_nothing_to_do(s2d2):
    b = au.Batch([(0, 10), (0, 0)], 4, 2, 64, spare=5)
    out, lse = b.attend(s2d2)
    assert (out == 7).all() and (lse == 7).all()
    kv = b.kv(s2d2)
    s2d2.paged_attention(0, 0, 4, s2d2.Rows(0, 2, 0, 0, 0, 3, 0), kv, 0, 0)
    s2d2.paged_attention(0, 0, 4, s2d2.Rows(5, 0, 0, 0, 0, 3, 1), kv, 0, 0)


def test_runs_are_equal_bit_for_bit(s2d2):
    b = au.Batch([(1, 3000), (70, 900), (8, 1500)], 8, 2, 128)
    first = b.attend(s2d2)
    for _ in range(5):
        again = b.attend(s2d2)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def test_captured_graph_runs_with_other_lengths_and_pages(s2d2):
    b = au.Batch([(2, 150), (1, 600), (3, 40)], 4, 2, 128)
    out, lse = torch.full((6, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((6, 4), 7.0, device="cuda")
    rows, kv = b.rows(s2d2), b.kv(s2d2)
    ws = torch.empty(s2d2.paged_attention_workspace(rows, kv, 4), dtype=torch.uint8, device="cuda")
    s2d2.ops_status()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s2d2.paged_attention(b.q_buf.data_ptr(), out.data_ptr(), 4, rows, kv, ws.data_ptr(), ws.numel(), d_lse=lse.data_ptr(),
                             stream=torch.cuda.current_stream().cuda_stream)
    for lens in ([(2, 150), (1, 600), (3, 40)], [(3, 20), (2, 599), (1, 3)], [(1, 1), (1, 64), (2, 38)]):
        short = [b.keys[s][:kv] for s, (_, kv) in enumerate(lens)], [b.values[s][:kv] for s, (_, kv) in enumerate(lens)]
        c = au.Batch.__new__(au.Batch)
        c.__dict__.update(b.__dict__, lens=lens, keys=short[0], values=short[1], first=[0, lens[0][0], lens[0][0] + lens[1][0], sum(n for n, _ in lens)])
        out.fill_(7), lse.fill_(7)
        b.row0.copy_(torch.tensor(c.first, dtype=torch.int32))
        b.kv_len.copy_(torch.tensor([kv for _, kv in lens], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        b.check((out, lse), c.want())


def test_two_streams_at_once_with_their_own_workspaces(s2d2):
    batches = [au.Batch([(1, 4000), (20, 500)], 8, 2, 128, seed=1), au.Batch([(300, 300), (1, 900)], 8, 2, 64, seed=2)]
    streams = [torch.cuda.Stream() for _ in batches]
    wants = [b.want() for b in batches]
    torch.cuda.synchronize()
    for _ in range(4):
        got = []
        for b, st in zip(batches, streams):
            with torch.cuda.stream(st):
                got.append(b.attend(s2d2))
        torch.cuda.synchronize()
        for b, g, w in zip(batches, got, wants):
            b.check(g, w)
