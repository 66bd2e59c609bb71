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
