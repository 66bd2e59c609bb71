"""Rows that are taken again one by one (a NaN in a value that they do not see): however long that takes, nothing that waits for it gives up."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


# an item for every CTA; heads shared by more CTAs than there are, with items behind the ones that are repaired; items of two tiles
@pytest.mark.parametrize("lens,heads,dim", [([(40, 8000)], 148, 64), ([(40, 6000), (3, 900), (40, 2500)], 60, 128), ([(200, 5000)], 100, 64)])
def test_waits_last_as_long_as_rows_are_repaired(s2d2, lens, heads, dim):
    """With a limit of some hundred microseconds for every wait, which the tiles keep, and repairs of many milliseconds."""
    from paper_2603_25702_b200 import binding
    stream = torch.cuda.current_stream().cuda_stream
    b = au.Batch(lens, heads, heads, dim)
    clean = b.want()
    limit = 64
    binding.debug_attention_wait(limit)
    got = b.attend(s2d2)
    s2d2.ops_status(stream)
    b.check(got, clean)
    for s, (n, kv) in enumerate(lens):
        if n >= 40:
            b.values[s][kv - 1] = float("nan")                       # the last row's own
    b.write()
    want = b.want()
    binding.debug_attention_wait(limit)
    got = b.attend(s2d2)
    s2d2.ops_status(stream)
    b.check(got, want)
    assert torch.isfinite(got[0][:lens[0][0] - 1]).all() and torch.isnan(got[0][lens[0][0] - 1]).all()


@pytest.mark.parametrize("lens,heads,kv_heads", [([(1, 100)], 2, 1), ([(3, 700)], 4, 2), ([(40, 300), (1, 5000)], 4, 2), ([(200, 500)], 2, 1)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("below", [20, 200, 4000])
def test_what_a_row_sees_counts_however_small_its_probability_is(s2d2, lens, heads, kv_heads, value, below):
    """A NaN or an infinity in one element of a value whose probability rounds to zero: that element is none of the numbers, the others are as ever."""
    b = au.Batch(lens, heads, kv_heads, 64)
    b.q.zero_()
    b.q[..., 0] = 1
    for s, (n, kv) in enumerate(lens):
        b.keys[s].zero_()
        b.keys[s][kv // 2, :, 0] = -below
    b.write()
    clean = b.want(0, scale=1.0)
    for s, (n, kv) in enumerate(lens):
        b.values[s][kv // 2, :, 9] = value
    b.write()
    out, lse = b.attend(s2d2, 0, scale=1.0)
    assert not torch.isfinite(out[..., 9]).any()
    out[..., 9] = clean[0][..., 9]
    clean[2][..., 9] = 1.0                                           # (replaced)
    b.check((out, lse), clean)


def test_rows_that_see_only_scores_of_minus_infinity_are_zero(s2d2):
    """Whatever their values hold: products of 3e38 and -3e38 are -inf."""
    b = au.Batch([(2, 150), (130, 140)], 2, 1, 64)
    b.q.zero_()
    b.q[..., 0] = 3e38
    for s in range(2):
        b.keys[s].zero_()
        b.keys[s][..., 0] = -3e38
        b.values[s][5:20, :, 3] = float("nan")
    b.write()
    out, lse = b.attend(s2d2)
    assert (out == 0).all() and torch.isneginf(lse).all()
