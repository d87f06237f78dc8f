"""A layer of experts at the ends of its ranges: groups of nearly 2^31 rows."""
import pytest
import torch

import plain_experts as X
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MOST = (1 << 31) - 1


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


@pytest.fixture(scope="module")
def longest():
    """2^31 - 1 rows of one column: whole numbers (x -1, 0 or 1; dy -1 or 1), and their turned form as one group without offsets."""
    x = torch.randint(-1, 2, (MOST,), device=DEV, generator=_gen(1), dtype=torch.int8)
    dy = torch.randint(0, 2, (MOST,), device=DEV, generator=_gen(2), dtype=torch.int8) * 2 - 1
    yield x, dy
    del x, dy
    torch.cuda.empty_cache()


# one group, and one that has nearly all of the rows behind a small one and an empty one
@pytest.mark.parametrize("bounds", [[0, MOST], [0, 5, 5, MOST]])
def test_turned_forms_and_weight_gradients_of_the_longest_groups(longest, bounds):
    off, E = _i32(bounds), len(bounds) - 1
    forms = []
    for v in longest:
        m = v.to(torch.bfloat16).view(MOST, 1)
        blocks = B.loka_grouped_blocks(MOST, E)
        qt, st = torch.full((blocks, 1, 128), 0xA5, dtype=torch.uint8, device=DEV), torch.full((blocks, 1), -7.0, device=DEV)
        B.loka_grouped_quantize(m, offsets=off, along=False, turned=True, qt=qt, st=st)
        at = 0
        for a, b in zip(bounds[:-1], bounds[1:]):
            if b > a:                   # against each group alone, without offsets (its rows are counted in 64 bits)
                one = B.loka_grouped_quantize(m[a:b], along=False, turned=True)
                n = len(one.qt)
                assert n == -(-(b - a) // 128) and torch.equal(qt[at:at + n], one.qt) and torch.equal(st[at:at + n], one.st)
                at += n
                del one
        assert bool((qt[at:] == 0xA5).all()) and bool((st[at:] == -7).all())
        c, f = X.turned(m[-1000:], [0, (1000 - (MOST - bounds[-2])) % 128, 1000])           # the last rows by the plain form
        assert torch.equal(X.e4m3(qt[at - 7:at]), c[-7:]) and torch.equal(st[at - 7:at].double(), f[-7:])
        forms += [qt, st]
        del m
    _, dw = B.loka_grouped_wgrad(B.make_grouped_desc(MOST, 1, 1, E), *forms, off, want_out=False, want_y=True)
    prod = longest[0] * longest[1]
    want = [int(prod[a:b].sum(dtype=torch.int64)) for a, b in zip(bounds[:-1], bounds[1:])]
    assert max(map(abs, want)) < 1 << 24 and dw.flatten().tolist() == want                   # (whole numbers below 2^24: exact)


@pytest.mark.parametrize("bounds", [[0, MOST], [0, 5, 5, MOST]])
def test_products_of_the_longest_groups(bounds):
    """2^31 - 1 rows, each one of 256 tokens of one element, times one column."""
    E = len(bounds) - 1
    x = torch.arange(-128, 128, device=DEV).to(torch.bfloat16).view(256, 1)
    x = torch.where(x.abs() > 16, x.sign() * 16, x)                                             # (whole numbers that 8 bits hold)
    index = torch.arange(MOST, device=DEV, dtype=torch.int32) & 255
    w = torch.arange(1, E + 1, device=DEV).to(torch.bfloat16).view(E, 1)
    wq = B.loka_grouped_quantize(w, groups=E, along=False, turned=True)
    out = torch.full((MOST, 1), -7.0, dtype=torch.bfloat16, device=DEV)
    B.loka_grouped_linear(B.make_grouped_desc(MOST, 1, 1, E), x, wq.qt, wq.st, _i32(bounds), index=index, out=out)
    del index
    head, tail = out[5:256].flatten(), out[256:-255].view(-1, 256)
    assert torch.equal(out[:5].flatten(), x[:5].flatten() * w[0]) and torch.equal(head, x[5:].flatten() * w[-1])
    assert bool((tail == x.flatten() * w[-1]).all()) and torch.equal(out[-255:].flatten(), x[:255].flatten() * w[-1])
    del out, head, tail
    torch.cuda.empty_cache()
