"""Parts of a shared cache whose references differ widely: scores that jump by almost the range of fp32 inside a tile of 128 keys, at any place of it.

Scores are set exactly: a query is the first unit vector, a key has its score (a power of two's exponent, with scale = ln 2) as its first element."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def check(s2d2, lens, heads, kv_heads, dim, levels, values, mask_block=1):
    """``levels`` and ``values`` [kv] of every sequence: the keys' scores, and factors of their values."""
    b = au.Batch(lens, heads, kv_heads, dim)
    b.q.zero_()
    b.q[..., 0] = 1
    for s, (x, f) in enumerate(zip(levels, values)):
        b.keys[s].zero_()
        b.keys[s][..., 0] = x[:, None].bfloat16()
        b.values[s].uniform_(0.25, 0.75).mul_(f[:, None, None].bfloat16())
    b.write()
    got = b.attend(s2d2, mask_block, scale=math.log(2))
    b.check(got, b.want(mask_block, scale=math.log(2)))
    s2d2.ops_status(torch.cuda.current_stream().cuda_stream)


def tiles(parts, gap, count, place, top):
    """Every other tile lies ``gap`` below ``top``, but for ``count`` keys from ``place`` on; in the others one key, the first, stands at 0."""
    x = torch.full((parts, 128), -60.0, device="cuda")
    x[:, 0] = 0
    x[::2] = top - gap
    x[::2, place:place + count] = top
    return x.flatten()


# (gap, keys at the top): their probabilities add up to at most 2^127.6 against the tile's first reference
JUMPS = [(80, 64), (99, 1), (101, 1), (110, 64), (120, 64), (121, 64), (126, 1), (127, 1), (127.5, 1)]


@pytest.mark.parametrize("parts", [1, 2, 4, 148, 601])
@pytest.mark.parametrize("gap,count", JUMPS)
@pytest.mark.parametrize("place", [40, 64, 127])
def test_a_jump_inside_a_part_beside_others(s2d2, parts, gap, count, place):
    """40: in a tile's first step, 64 and 127: in its second, behind which a CTA of one tile has none."""
    count = min(count, 128 - place)
    for top in (1.0, 0.0):
        x = tiles(parts, gap, count, place, top)
        check(s2d2, [(1, 128 * parts)], 2, 1, 64, [x], [torch.ones_like(x)])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("gap,count", JUMPS)
def test_a_jump_at_the_end_of_items_of_one_and_of_two_tiles(s2d2, dim, gap, count):
    """Whole items and shared ones, rows that end in front of, in and behind the jump."""
    lens = [(1, 128), (3, 512), (200, 640), (1, 1500)]
    x = [tiles(-(-kv // 128), gap, count, 64, 1.0)[:kv] for _, kv in lens]
    f = [torch.ones_like(t) for t in x]
    check(s2d2, lens, 4, 2, dim, x, f)
    check(s2d2, lens[:2], 4, 2, dim, x[:2], f[:2], 0)


@pytest.mark.parametrize("n", [1, 200])
def test_many_high_parts_do_not_add_up_to_infinity(s2d2, n):
    """512 keys, half of them 121 above the first of their tile: each part's sum is 2^127."""
    x = torch.zeros(4, 128, device="cuda")
    x[:, 64:] = 121
    check(s2d2, [(n, 512)], 1, 1, 64, [x.flatten()], [torch.ones(512, device="cuda")], 0)


@pytest.mark.parametrize("low,high", [(-126.5, 1.0), (-127, 0.5), (-127, 0.75)])
def test_a_part_far_below_another_reference_keeps_its_weight(s2d2, low, high):
    """Two parts of about equal weight whose first references are more than 126 apart; the values tell them apart."""
    x = torch.full((2, 128), -200.0, device="cuda")
    x[0] = low
    x[0, 100] = high
    x[1, 0] = 0
    f = torch.ones(256, device="cuda")
    f[100] = -1
    check(s2d2, [(1, 256)], 2, 1, 64, [x.flatten()], [f])
