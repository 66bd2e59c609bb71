"""Lists of rows that decrease: whose rows the append writes."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def owners(row0, n_rows):
    """[(first, end)] of each sequence's rows, None where it has none."""
    return [(a, e) if 0 <= a < e <= n_rows else None for a, e in zip(row0, row0[1:])]


def set_list(b, row0):
    b.row0.copy_(torch.tensor(row0, dtype=torch.int32))


def alone(b, s, rows):
    """A list in which sequence s has these rows and no other has any."""
    set_list(b, [rows[0]] * (s + 1) + [rows[1]] * (len(b.lens) - s))


# ends of zeros, entries out of range between good ones, idle sequences
FOLLOWED = [[0, 4, 8, 0, 0, 0, 0], [0, 4, -1, 4, 8, 8, 8], [0, 4, 200, 4, 8, 8, 16], [3, 3, 0, 8, 8, 9, 100], [0, 2 ** 31 - 1, 0, 6, -2 ** 31, 6, 14]]
UNORDERED = [[4, 8, 0, 4, 4, 4, 4], [50, 58, 58, 10, 18, 0, 8]]
OVERLAPPING = [[0, 8, 4, 12, 12, 12, 12], [0, 30, 10, 40, 40, 40, 40], [8, 16, 0, 9, 9, 9, 9], [0, 8, 8, 16, 15, 20, 20], [0, 40, 39, 40, 40, 0, 1]]


def append(s2d2, b, x, rope, empty):
    """(cache, q_out) behind an append to ``empty``."""
    b.cache.copy_(empty)
    q_out = torch.full((b.n_rows, 2 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    s2d2.kv_append(x[:, 128:].data_ptr(), x[:, 192:].data_ptr(), "fp32", b.rows(s2d2), b.kv(s2d2), rope, k_stride=256, v_stride=256, d_q=x.data_ptr(),
                   d_q_out=q_out.data_ptr(), n_q_heads=2, q_stride=256, stream=torch.cuda.current_stream().cuda_stream)
    return b.cache.clone(), q_out


def setup(s2d2, lens, spare):
    b = au.Batch(lens, 2, 1, 64, page=16, spare=spare, poison=5.0)
    x = torch.randn(b.n_rows, 256, device="cuda")
    freqs = au.frequencies(64).cuda()
    return b, x, s2d2.Rope(freqs.data_ptr(), 64), b.cache.clone(), freqs


@pytest.mark.parametrize("row0", FOLLOWED + UNORDERED)
def test_append_finds_the_rows_of_every_sequence_that_has_some(s2d2, row0):
    b, x, rope, empty, _freqs = setup(s2d2, [(8, 60 + 9 * s) for s in range(6)], 52)
    cache, q = empty.clone(), torch.full((100, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    for s, rows in enumerate(owners(row0, b.n_rows)):
        if rows:
            alone(b, s, rows)
            c, q_one = append(s2d2, b, x, rope, empty)
            cache = torch.where(c != empty, c, cache)
            q[rows[0]:rows[1]] = q_one[rows[0]:rows[1]]
    assert (q != 7).any()
    set_list(b, row0)
    got = append(s2d2, b, x, rope, empty)
    assert torch.equal(got[1], q) and torch.equal(got[0], cache)


@pytest.mark.parametrize("row0", OVERLAPPING)
def test_append_gives_a_row_of_several_sequences_to_one_of_them(s2d2, row0):
    b, x, rope, empty, _freqs = setup(s2d2, [(8, 60 + 9 * s) for s in range(6)], 52)
    matches = torch.zeros(100, dtype=torch.bool, device="cuda")
    has = torch.zeros(100, dtype=torch.bool, device="cuda")
    ones = []
    for s, rows in enumerate(owners(row0, b.n_rows)):
        if rows:
            alone(b, s, rows)
            ones.append((rows, append(s2d2, b, x, rope, empty)[1]))
    set_list(b, row0)
    _, q = append(s2d2, b, x, rope, empty)
    for (a, e), one in ones:
        matches[a:e] |= (q[a:e] == one[a:e]).all(1)
        has[a:e] = True
    assert torch.equal(matches, has) and (q[~has] == 7).all()


def test_append_to_many_sequences_with_an_end_of_zeros(s2d2):
    b, x, rope, empty, _freqs = setup(s2d2, [(1, 20 + s % 30) for s in range(700)], 60)
    want = append(s2d2, b, x, rope, empty)
    row0 = list(range(701))
    set_list(b, row0[:650] + [649] * 51)
    want = append(s2d2, b, x, rope, empty)
    set_list(b, row0[:650] + [0] * 51)
    got = append(s2d2, b, x, rope, empty)
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and not torch.equal(want[0], empty)
