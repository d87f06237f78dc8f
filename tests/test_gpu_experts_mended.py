"""A layer of experts: calls that are documented and were once answered wrongly or refused, or took a form that no test reached."""
import math

import pytest
import torch

import plain_experts as X
import plain_ops as P
import test_gpu_experts as G
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


@pytest.mark.parametrize("T,k,C", [(40, 3, 7), (33, 8, 257), (5, 2, 1001), (3, 4, 4095), (8200, 4, 4099)])
def test_combination_of_matrices_that_start_anywhere(T, k, C):
    """Rows from the second on of matrices of odd width, which no 16 bytes divide, against the same rows at aligned places."""
    rows = T * k
    y, res, dout = (_randn(n + 1, C, seed=i).bfloat16()[1:] for i, n in enumerate((rows, T, T)))
    slots = torch.randperm(rows, device=DEV, generator=_gen(3)).view(T, k).int()
    w = _randn(T, k, seed=4)
    apart = [t.clone() for t in (y, res, dout)]
    assert all(a.data_ptr() % 16 == 0 and t.data_ptr() % 16 for a, t in zip(apart, (y, res, dout)))
    want = B.loka_combine(apart[0], slots, w, apart[1])
    out = torch.full((T + 2, C), -7.0, dtype=torch.bfloat16, device=DEV)
    assert torch.equal(B.loka_combine(y, slots, w, res, out=out[1:T + 1]), want) and bool((out[0] == -7).all()) and bool((out[T + 1] == -7).all())
    dy0, dw0 = B.loka_combine_backward(apart[2], apart[0], slots, w)
    dy = torch.full((rows + 2, C), -7.0, dtype=torch.bfloat16, device=DEV)
    _, dw = B.loka_combine_backward(dout, y, slots, w, dy=dy[1:rows + 1])
    assert torch.equal(dy[1:rows + 1], dy0) and torch.equal(dw, dw0) and bool((dy[0] == -7).all()) and bool((dy[rows + 1] == -7).all())
    assert torch.equal(B.loka_combine(y, slots, w, res, out=res), want)             # over the residual


@pytest.mark.parametrize("T", [16384, 140000])
def test_quantize_many_gathered_rows(T):
    """2^27 elements and more of a source that the cache holds, and of one that it does not: both read the same rows."""
    C, rows = 1024, 140000
    x = torch.randn(T, C, device=DEV, generator=_gen(T), dtype=torch.bfloat16)
    index = torch.randint(0, T, (rows,), device=DEV, generator=_gen(1)).int()
    bounds = [0, 70001, 70001, rows]
    r = B.loka_grouped_quantize(x, offsets=_i32(bounds), index=index, turned=True)
    alone = B.loka_grouped_quantize(x, offsets=_i32(bounds), index=index)
    only = B.loka_grouped_quantize(x, offsets=_i32(bounds), index=index, along=False, turned=True)
    used = 547 + 547                    # blocks of 70001 and 69999 rows
    assert torch.equal(alone.q, r.q) and torch.equal(alone.scales, r.scales)
    assert torch.equal(only.qt[:used], r.qt[:used]) and torch.equal(only.st[:used], r.st[:used])
    for a, b, block in ((0, 1280, 0), (69888, 70001, 546), (70001, 70001 + 1280, 547), (70001 + 546 * 128, rows, 1093)):
        v = x[index[a:b].long()]
        c, f = X.along(v)
        assert torch.equal(X.e4m3(r.q[a:b]), c) and torch.equal(r.scales[a:b].double(), f)
        c, f = X.turned(v, [0, b - a])
        assert torch.equal(X.e4m3(r.qt[block:block + len(c)]), c) and torch.equal(r.st[block:block + len(c)].double(), f)


# (tokens, experts, choices, score, renorm, bf16): chunks of 16 to 128 tokens, below and above the number from which their counts have a launch of their own,
# with every number of lanes a token; test_experts_launches.py holds them to that
@pytest.mark.parametrize("T,E,k,score,renorm,bf16", [
    (1000, 1024, 16, "sigmoid", True, False), (2000, 200, 3, "softmax", False, True), (4097, 64, 2, "softmax", True, True), (8192, 300, 3, "sigmoid", False, False),
    (8193, 100, 9, "softmax", True, False), (16384, 1000, 2, "softmax", False, True), (16385, 256, 8, "sigmoid", True, True), (32768, 256, 8, "softmax", True, True),
    (32700, 33, 5, "sigmoid", False, False), (32769, 1024, 4, "sigmoid", True, False), (40000, 512, 6, "softmax", False, True), (33000, 160, 16, "sigmoid", False, False),
    (50001, 128, 1, "softmax", True, True), (66000, 7, 7, "sigmoid", True, True)])
def test_route_sizes(T, E, k, score, renorm, bf16):
    x = 1.5 * _randn(T, E, seed=T)
    x[:, E // 3] += 3.0                 # an expert that most tokens take
    x[torch.rand(T, E, device=DEV, generator=_gen(1)) < 0.3] = -math.inf
    x[5:9] = -math.inf                  # tokens that choose nothing
    x = x.bfloat16() if bf16 else x
    r = B.loka_route(x, k, G.SCORES[score], renorm, 2.5)
    e = X.choose(x, k)
    assert torch.equal(r.experts.long(), e)
    slots, rows, offsets = X.order_of_many(e, E)
    assert torch.equal(r.slots, slots) and torch.equal(r.rows, rows) and torch.equal(r.offsets, offsets)
    # counted as in test_gpu_experts._check_route
    w = torch.where(e >= 0, X.weights(x, e, score, renorm, 2.5), 0.0)
    span = float(torch.where(x.isfinite(), x.double(), 0.0).abs().max())
    assert bool(((r.weights.double() - w).abs() <= (2 * (2 * span + 4) + 24 + 6) * P.F32 * w + 2.0 ** -126).all())
    # the gradient: the formulas in 64 bits
    g = _randn(T, k, seed=2)
    got = B.loka_route_backward(x, r.experts, g, G.SCORES[score], renorm, 2.5)
    live = e >= 0
    gd, at = torch.where(live, 2.5 * g.double(), 0.0), e.clamp_min(0)
    q = w / 2.5
    sig = torch.sigmoid(x.double().gather(1, at))
    want = torch.zeros(T, E, dtype=torch.float64, device=DEV)
    inner = (gd * q).sum(1, keepdim=True)
    if score == "softmax" and not renorm:
        want = -torch.nan_to_num(torch.softmax(x.double(), 1)) * inner
        d = gd * q
    elif renorm:
        d = q * (gd - inner) * (1 - sig if score == "sigmoid" else 1.0)
    else:
        d = gd * sig * (1 - sig)
    want.scatter_add_(1, at, torch.where(live, d, 0.0))
    # counted as in test_gpu_experts.test_route_backward, of logits up to `span`
    tol = (2 * (2 * span + 4) + 24 + 16 + 8) * P.F32 * 2.5 * float(g.abs().max()) * 2
    assert bool(((got.double() - want).abs() <= tol + (G.BF * want.abs() if bf16 else 0.0)).all()) and not bool(got[5:9].any())


@pytest.mark.parametrize("sizes", [[200 + (i * 37) % 11 * 40 for i in range(100)]])
def test_weight_gradients_of_many_groups(sizes):
    """More than 64 groups in large tiles."""
    G.test_weight_gradients_are_exact_on_whole_numbers(sizes, 1008, 720)


@pytest.mark.parametrize("sizes,K,N", G.FORMS[:-1] + [([1], 4096, 1000), ([3, 0, 5], 513, 40)])
def test_the_linear_is_the_quantization_and_the_product(sizes, K, N):
    """The same bits, in every form of the product."""
    n, E = sum(sizes), len(sizes)
    off = _i32([0] + torch.tensor(sizes).cumsum(0).tolist())
    x, w = _randn(max(5, n // 2), K, seed=K).bfloat16(), (_randn(E * K, N, seed=N) / math.sqrt(K)).bfloat16()
    x[:, ::17] *= 20.0
    index = torch.randint(0, len(x), (n,), device=DEV, generator=_gen(n)).int()
    wq = B.loka_grouped_quantize(w, groups=E, along=False, turned=True)
    d = B.make_grouped_desc(n, N, K, E)
    out, y = B.loka_grouped_linear(d, x, wq.qt, wq.st, off, index=index, want_y=True)
    xq = B.loka_grouped_quantize(x)
    o2, y2 = B.loka_grouped_gemm(d, xq.q, xq.scales, wq.qt, wq.st, off, index=index, want_y=True)
    xg = x[index.long()]
    o3, y3 = B.loka_grouped_linear(d, xg, wq.qt, wq.st, off, want_y=True)
    assert torch.equal(y, y2) and torch.equal(out, o2) and torch.equal(y, y3) and torch.equal(out, o3) and torch.equal(out, y.bfloat16())
