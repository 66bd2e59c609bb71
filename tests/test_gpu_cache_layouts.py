"""Append and attention on caches with pages, heads and tokens inside one another in every order."""
import itertools

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


def lay_out(b, order, shared):
    """The batch's keys and values in [order[0]][order[1]][order[2]][element], both in one buffer (outside of all, or beside each head's elements) or not."""
    size = {"page": b.n_pages, "head": b.kv_heads, "token": b.page}
    shape = [size[name] for name in order]
    if shared == "outside":
        both = torch.full([2] + shape + [b.dim], float("nan"), dtype=torch.bfloat16, device="cuda")
    elif shared == "beside":
        both = torch.full(shape + [2, b.dim], float("nan"), dtype=torch.bfloat16, device="cuda").movedim(3, 0)
    else:
        both = [torch.full(shape + [b.dim + 8], float("nan"), dtype=torch.bfloat16, device="cuda")[..., :b.dim] for _ in range(2)]
    place = [order.index(name) for name in ("page", "head", "token")] + [3]
    b.cache, b.k, b.v = both[0], both[0].permute(place), both[1].permute(place)
    return both


@pytest.mark.parametrize("order", list(itertools.permutations(["page", "head", "token"])))
@pytest.mark.parametrize("shared", ["outside", "beside", "no"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 128), (40, 64)])
def test_append_and_attention(s2d2, order, shared, dim, page):
    b = au.Batch([(1, 300), (70, 260), (0, 4), (3, 3)], 6, 3, dim, page=page)
    both = lay_out(b, order, shared)
    kv = [torch.cat([t[s][b.lens[s][1] - b.lens[s][0]:] for s in range(4)]) for t in (b.keys, b.values)]       # the new rows'
    b.write()
    for s, (n, length) in enumerate(b.lens):
        where, tok = (t[length - n:] for t in b.places(s))
        b.k.transpose(1, 2)[where, tok] = b.v.transpose(1, 2)[where, tok] = 9.0
    s2d2.kv_append(kv[0].data_ptr(), kv[1].data_ptr(), "bf16", b.rows(s2d2), b.kv(s2d2), stream=torch.cuda.current_stream().cuda_stream)
    for s in range(4):
        where, tok = b.places(s)
        assert torch.equal(b.k.transpose(1, 2)[where, tok], b.keys[s]) and torch.equal(b.v.transpose(1, 2)[where, tok], b.values[s])
    used = sum(length for _, length in b.lens) * 3 * dim * 2
    assert sum(int((~torch.isnan(t)).sum()) for t in both) == used                                             # and nothing else was written
    b.check(b.attend(s2d2), b.want())
