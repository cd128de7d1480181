"""Overlaps of arrays whose sizes pass 64 bits, as the loss on stored logits refuses them (CPU: addresses are never read)."""
from paper_2605_07230_b200 import binding as cb
from tests.test_distill_refusals import AT, grad, loss


def test_products_of_sizes_past_64_bits():
    """Arrays of 2^31 rows of 2^31 entries reach over everything behind them."""
    most = 2**31 - 1
    assert loss(K=most, n=2**31 - 65536, h=most, top=0x10000000, loss=0x20000000) == cb.ERR_INVALID_ARG
    assert grad(K=most, n=2**31 - 65536, ids=AT["top"], grad=AT["up"]) == cb.ERR_INVALID_ARG
