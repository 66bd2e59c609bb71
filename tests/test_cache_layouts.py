"""Orders of the dimensions of a paged cache: any that nests is taken, with or without a GPU to run on."""
import itertools

import pytest

P = 1 << 20     # a pointer value that no check may follow
SIZES = {"page": 6, "head": 3, "token": 16}


@pytest.fixture(scope="module")
def s2d2():
    from paper_2603_25702_b200.build import build
    build()
    import paper_2603_25702_b200 as m
    return m


def strides(order, dim, sizes=SIZES, gap=0):
    """Strides of [order[0]][order[1]][order[2]][element]."""
    out, at = {}, dim + gap
    for name in reversed(order):
        out[name] = at
        at = at * sizes[name] + gap
    return out


def kv(s2d2, st, dim=64, sizes=SIZES):
    return s2d2.PagedKV(P, P, sizes["page"], sizes["token"], sizes["head"], dim, page_stride=st["page"], head_stride=st["head"], token_stride=st["token"])


def needs(s2d2, c, heads=6):
    return s2d2.paged_attention_workspace(s2d2.Rows(8, 2, P, P, P, 3), c, heads)


@pytest.mark.parametrize("order", list(itertools.permutations(SIZES)))
@pytest.mark.parametrize("gap", [0, 8])
def test_every_order_is_taken(s2d2, order, gap):
    assert needs(s2d2, kv(s2d2, strides(order, 64, gap=gap))) > 0


@pytest.mark.parametrize("order", list(itertools.permutations(SIZES)))
@pytest.mark.parametrize("inner", range(3))
def test_overlap_is_refused_in_every_order(s2d2, order, inner):
    """A stride one step too short for what is inside of it."""
    st = strides(order, 64)
    st[order[inner]] -= 8
    with pytest.raises(s2d2.S2D2Error) as e:
        needs(s2d2, kv(s2d2, st))
    assert e.value.code == -1 and "overlap" in str(e.value)


@pytest.mark.parametrize("one", ["page", "head"])
def test_the_stride_of_a_single_page_or_head_does_not_matter(s2d2, one):
    sizes = {**SIZES, one: 1}
    for order in itertools.permutations(SIZES):
        st = strides(order, 64, sizes)
        st[one] = 8
        assert needs(s2d2, kv(s2d2, st, sizes=sizes), 2 * sizes["head"]) > 0


def test_the_largest_strides_do_not_wrap(s2d2):
    """Spans beyond 64 bits: 2^31 - 1 pages 2^38 elements apart, with heads inside and outside of them."""
    big = {"page": 2 ** 31 - 1, "head": 2, "token": 16}
    assert needs(s2d2, kv(s2d2, {"page": 1 << 38, "head": 1024, "token": 64}, sizes=big), 4) > 0
    for head in (1 << 38, (1 << 38) - 8):
        with pytest.raises(s2d2.S2D2Error) as e:
            needs(s2d2, kv(s2d2, {"page": 1 << 38, "head": head, "token": 64}, sizes=big), 4)
        assert "overlap" in str(e.value)


@pytest.mark.parametrize("dim", [0, -8, 2 ** 40, 12])
def test_a_head_size_that_is_none_is_refused_like_any_other(s2d2, dim):
    """With the scale that follows from it left out, too."""
    with pytest.raises(s2d2.S2D2Error) as e:
        s2d2.paged_attention(P, P, 6, s2d2.Rows(8, 2, P, P, P, 3), kv(s2d2, strides(("page", "head", "token"), 64), dim), P, 1 << 40)
    assert e.value.code == -1 and "head_dim" in str(e.value)
