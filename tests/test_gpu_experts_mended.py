"""A layer of experts: calls that are documented and were once answered wrongly or refused, or took a form that no test reached."""
import pytest
import torch

import plain_experts as X
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(*shape, seed):
    return torch.randn(*shape, device=DEV, generator=_gen(seed))


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_a_buffer_that_is_given_is_written():
    """... whether or not its form was asked for."""
    x = _randn(300, 200, seed=1).bfloat16()
    want = B.loka_grouped_quantize(x, turned=True)
    q, s, qt, st = (torch.empty_like(t) for t in want)
    for t in (q, s, qt, st):
        t.fill_(3)
    r = B.loka_grouped_quantize(x, qt=qt, st=st)
    assert r.qt.data_ptr() == qt.data_ptr() and all(torch.equal(a, b) for a, b in zip(r, want))
    r = B.loka_grouped_quantize(x, along=False, turned=True, q=q, scales=s)
    assert r.q.data_ptr() == q.data_ptr() and all(torch.equal(a, b) for a, b in zip(r, want))
    for name in ("q", "scales", "qt", "st"):       # one of a pair: the other one is new
        one = torch.empty_like(getattr(want, name))
        r = B.loka_grouped_quantize(x, along=False, turned=False, **{name: one})
        assert getattr(r, name).data_ptr() == one.data_ptr() and torch.equal(one, getattr(want, name))
        assert [t is None for t in r] == ([False, False, True, True] if name in ("q", "scales") else [True, True, False, False])
