"""Lists of rows that decrease: which of their sequences the attention follows."""
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


@pytest.mark.parametrize("row0", FOLLOWED)
@pytest.mark.parametrize("max_rows", [8, 100])
def test_attention_follows_a_list_whose_sequences_come_in_the_order_of_their_rows(s2d2, row0, max_rows):
    b = au.Batch([(8, 100)] * 6, 4, 2, 64, spare=52)
    want = [torch.full((100, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((100, 4), 7.0, device="cuda")]
    for s, rows in enumerate(owners(row0, b.n_rows)):
        if rows:
            alone(b, s, rows)
            for w, g in zip(want, b.attend(s2d2)):
                w[rows[0]:rows[1]] = g[rows[0]:rows[1]]
    set_list(b, row0)
    out, lse = b.attend(s2d2, max_rows=max_rows)
    assert torch.equal(out == 7, want[0] == 7) and torch.equal(lse == 7, want[1] == 7)
    # (cut into other parts: sums of at most 100 keys in another order, probabilities rounded otherwise, one rounding of the output each)
    size = 4.0                                                       # of a value
    assert ((out.float() - want[0].float()).abs() <= size * (2.0 ** -8 + 100 * 2.0 ** -23) + 2 * want[0].float().abs() * 2.0 ** -8).all()
    assert ((lse - want[1]).abs() <= 2.0 ** -15).all()


@pytest.mark.parametrize("row0", UNORDERED + OVERLAPPING)
@pytest.mark.parametrize("max_rows", [8, 100])
def test_attention_follows_no_other_list(s2d2, row0, max_rows):
    """Padded: the rows of all sequences together are fewer than those of the batch."""
    b = au.Batch([(8, 100)] * 6, 4, 2, 64, spare=52)
    set_list(b, row0)
    out, lse = b.attend(s2d2, max_rows=max_rows)
    assert (out == 7).all() and (lse == 7).all()


@pytest.mark.parametrize("at", [1, 31, 32, 33, 70, 98])
def test_attention_of_many_sequences_with_one_that_begins_too_early(s2d2, at):
    b = au.Batch([(1, 40)] * 100, 2, 1, 64, spare=200)
    row0 = list(range(101))
    row0[at] = 0                                                     # at: a sequence of rows 0 .. at
    set_list(b, row0)
    out, lse = b.attend(s2d2, max_rows=100)
    if at == 1:                                                      # this one does not decrease: 0 has no rows, 1 has two
        assert (out[:100] != 7).any(2).all() and (out[100:] == 7).all() and (lse[:100] != 7).all() and (lse[100:] == 7).all()
    else:
        assert (out == 7).all() and (lse == 7).all()
    row0[at] = -1                                                    # at - 1 and at have none
    set_list(b, row0)
    out, lse = b.attend(s2d2, max_rows=100)
    idle = torch.ones(300, dtype=torch.bool, device="cuda")
    idle[:100] = False
    idle[at - 1:at + 1] = True
    assert torch.equal((lse == 7).all(1), idle) and torch.equal((out == 7).all(2).all(1), idle)
