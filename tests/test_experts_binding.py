"""A layer of experts without a GPU: what the binding makes of its arguments."""
import pytest
import torch

import plain_experts as X
from paper_2605_10886_amd import binding as B


def test_a_buffer_that_is_given_asks_for_its_form():
    x, u, f = torch.zeros(8, 16, dtype=torch.bfloat16), torch.zeros(16, 128, dtype=torch.uint8), torch.zeros(16)
    for kw in (dict(q=u), dict(scales=f), dict(qt=u), dict(st=f)):
        with pytest.raises(AssertionError, match="one GPU"):            # (past "one of the two forms at least")
            B.loka_grouped_quantize(x, along=False, **kw)


def test_the_two_plain_orders_agree():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(200, 9, generator=g)
    x[torch.rand(200, 9, generator=g) < 0.6] = -float("inf")
    e = X.choose(x, 4)
    assert bool((e < 0).any()) and all(torch.equal(a, b) for a, b in zip(X.order(e, 9), X.order_of_many(e, 9)))
