"""How probabilities are rounded for the product with the values: which of them to twice the bits, on sums that show it exactly."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from tests import attention_util as au  # noqa: E402


@pytest.fixture(scope="module")
def s2d2():
    import paper_2603_25702_b200 as m
    return m


# max_rows * heads / kv_heads is at most 128; whole items and parts of shared ones
@pytest.mark.parametrize("lens,max_rows", [([(1, 128)], 1), ([(1, 1500)], 1), ([(16, 1222)] * 12, 16), ([(16, 300), (1, 20000)], 16), ([(20, 512)], 20)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("exponent", [-0.875, -1.25, -3.375])
def test_the_first_32_keys_of_64_lose_nothing_where_rows_are_few(s2d2, lens, max_rows, dim, exponent):
    """The first key of each tile of 128 has score 0 and value 0, all others the same score and, the first 32 of every 64, the same values: their
    probabilities have the same rounding error d, up to 2^-8, and so has the output without its remainder.  With it d is 2^-16; at most 400 additions of
    equal terms in fp32, one behind the other (a tile takes 16 and 8, a CTA has at most 14), are off by 2^-23 each; the exponential and the division are small
    beside that: 2^-14 in all, and the output's own rounding."""
    b = au.Batch(lens, 8, 2, dim)
    b.q.zero_()
    b.q[..., 0] = 1
    level = torch.linspace(1, 2, dim, device="cuda").bfloat16()
    for s, (_, kv) in enumerate(lens):
        b.keys[s].zero_()
        b.keys[s][:, :, 0] = exponent                                # (a bf16 number)
        b.keys[s][::128, :, 0] = 0
        b.values[s].zero_()
        b.values[s][torch.arange(kv, device="cuda") % 64 < 32] = level
        b.values[s][::128] = 0
    b.write()
    want = b.want(0, scale=math.log(2))[0]
    out = b.attend(s2d2, 0, scale=math.log(2), max_rows=max_rows)[0].double()
    half = 2.0 ** (torch.floor(torch.log2(want)) - 8)                # half a step of bf16
    assert ((out - want).abs() <= half + want * 2.0 ** -14).all()
    p = torch.tensor(2.0 ** exponent)
    assert (p.bfloat16() - p).abs() / p > 0.6 * 2.0 ** -9            # which would not have gone unseen
