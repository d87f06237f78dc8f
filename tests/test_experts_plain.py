"""A layer of experts without a GPU: what its entry points refuse before any HIP call, and the plain forms that the GPU tests compare
with, against differences."""
import ctypes

import pytest
import torch

import plain_experts as X
from paper_2605_10886_amd import binding as B

FAKE, ODD, OTHER = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0x1008)
SHAPE, NULL, ALIGN, UNSUPPORTED, WORKSPACE = B.LOKA_ERR_SHAPE, B.LOKA_ERR_NULL, B.LOKA_ERR_ALIGN, B.LOKA_ERR_UNSUPPORTED, B.LOKA_ERR_WORKSPACE
MOST = (1 << 31) - 1
ref = ctypes.byref


def _route_desc(tokens=4, ld=8, experts=8, top_k=2, score=B.SCORE_SOFTMAX, renorm=1, bf16=0, scale=1.0):
    return B.RouteDesc(tokens, ld, experts, top_k, score, renorm, bf16, scale)


def test_route_refusals():
    names = ("logits", "expert", "weight", "slot", "row", "offsets")

    def call(d, ws=None, nws=0, **kw):
        return B.lib().loka_route(ref(d), *[kw.get(n, FAKE) for n in names], ws, nws, None)

    def back(d, **kw):
        return B.lib().loka_route_backward(ref(d), *[kw.get(n, FAKE) for n in ("logits", "expert", "dweight", "dlogits")], None)

    for n in names:
        assert call(_route_desc(), **{n: None}) == NULL and call(_route_desc(), **{n: ODD}) == ALIGN
    for n in ("logits", "expert", "dweight", "dlogits"):
        assert back(_route_desc(), **{n: None}) == NULL and back(_route_desc(), **{n: ODD}) == ALIGN
    for kw in (dict(tokens=0), dict(tokens=-1), dict(tokens=(1 << 25) + 1), dict(experts=0), dict(experts=1025, ld=2000), dict(ld=7), dict(top_k=0),
               dict(top_k=9), dict(top_k=17, experts=64, ld=64), dict(tokens=1 << 25, ld=1 << 24)):
        assert call(_route_desc(**kw)) == SHAPE and back(_route_desc(**kw)) == SHAPE, kw
        assert B.lib().loka_route_workspace(ref(_route_desc(**kw))) == 0
    for score in (-1, 2):
        assert call(_route_desc(score=score)) == back(_route_desc(score=score)) == UNSUPPORTED
    many = _route_desc(tokens=100000)
    need = B.lib().loka_route_workspace(ref(many))
    assert need > 0 and call(many) == call(many, ws=FAKE, nws=need - 1) == WORKSPACE and call(many, ws=OTHER, nws=need) == ALIGN


def test_grouped_quantize_refusals():
    def call(x=FAKE, index=None, offsets=None, q=FAKE, s=FAKE, qt=None, st=None, rows=8, cols=16, ld=16, x_rows=8, groups=2):
        return B.lib().loka_grouped_quantize(ref(B.GroupedQuantizeDesc(rows, cols, ld, x_rows, groups)), x, index, offsets, q, s, qt, st, None)

    assert call(x=None) == call(q=None) == call(s=None) == call(qt=FAKE) == call(st=FAKE) == call(q=None, s=None) == NULL
    for kw in (dict(rows=0), dict(rows=MOST + 1), dict(cols=0), dict(cols=(1 << 20) + 1, ld=1 << 21), dict(ld=15), dict(groups=0), dict(groups=1025, rows=1025),
               dict(groups=3), dict(index=FAKE, x_rows=0), dict(index=FAKE, x_rows=MOST + 1), dict(rows=MOST, cols=1 << 20, ld=1 << 20, groups=1)):
        assert call(**kw) == SHAPE, kw
    for n in ("x", "index", "offsets", "q", "s"):
        assert call(**{n: ODD}) == ALIGN, n
    assert call(qt=ODD, st=FAKE) == call(qt=FAKE, st=ODD) == ALIGN
    blocks = B.loka_grouped_blocks
    assert [blocks(*a) for a in ((0, 1), (1, 0), (1, 1025), (MOST + 1, 1), (1, 1), (1, 64), (128, 1), (129, 1), (129, 2), (256, 256))] == [-1, -1, -1, -1, 1, 1, 1, 2, 2, 256]
    for rows, groups in ((1, 1), (7, 3), (300, 5), (300, 300), (1000, 7)):         # enough for any sizes: the worst is one row in every group but one
        some = min(rows, groups)
        assert blocks(rows, groups) >= some - 1 + -(-(rows - some + 1) // 128)


def test_grouped_product_refusals():
    def desc(rows=8, x_rows=8, N=16, K=16, groups=2, w_form=B.W_TURNED):
        return B.GroupedDesc(rows, x_rows, N, K, groups, w_form)

    def gemm(d, index=None, xq=FAKE, sx=FAKE, offsets=FAKE, wq=FAKE, sw=FAKE, out=FAKE, y=None):
        return B.lib().loka_grouped_gemm(ref(d), xq, sx, index, offsets, wq, sw, out, y, None)

    def linear(d, index=None, x=FAKE, ld=16, offsets=FAKE, wq=FAKE, sw=FAKE, out=FAKE, y=None, ws=FAKE, nws=1 << 40):
        return B.lib().loka_grouped_linear(ref(d), x, ld, index, offsets, wq, sw, out, y, ws, nws, None)

    def wgrad(d, xt=FAKE, sxt=FAKE, dyt=FAKE, sdyt=FAKE, offsets=FAKE, out=FAKE, y=None, ws=None, nws=0):
        return B.lib().loka_grouped_wgrad(ref(d), xt, sxt, dyt, sdyt, offsets, out, y, ws, nws, None)

    for n in ("xq", "sx", "offsets", "wq", "sw", "out"):
        assert gemm(desc(), **{n: None}) == NULL and gemm(desc(), **{n: ODD}) == ALIGN, n
    for n in ("x", "offsets", "wq", "sw", "out"):
        assert linear(desc(), **{n: None}) == NULL and linear(desc(), **{n: ODD}) == ALIGN, n
    for n in ("xt", "sxt", "dyt", "sdyt", "offsets", "out"):
        assert wgrad(desc(), **{n: None}) == NULL and wgrad(desc(), **{n: ODD}) == ALIGN, n
    assert gemm(desc(), y=ODD) == gemm(desc(), index=ODD) == linear(desc(), y=ODD) == linear(desc(), index=ODD) == wgrad(desc(), y=ODD) == ALIGN
    wide = (1 << 20) + 1
    for kw in (dict(rows=0), dict(rows=MOST + 1), dict(N=0), dict(N=wide), dict(K=0), dict(K=wide), dict(groups=0), dict(groups=1025), dict(rows=MOST, N=1 << 20)):
        assert gemm(desc(**kw)) == linear(desc(**kw), ld=1 << 21) == SHAPE, kw
        assert B.lib().loka_grouped_linear_workspace(ref(desc(**kw)), 0) == 0
        if kw != dict(rows=MOST, N=1 << 20):
            assert wgrad(desc(**kw)) == SHAPE and B.lib().loka_grouped_wgrad_workspace(ref(desc(**kw))) == 0
    assert wgrad(desc(N=1 << 20, K=1 << 20)) == SHAPE
    long = desc(rows=1 << 20, N=64, K=64, groups=1)                                # few results, a long sum: partial sums
    need = B.lib().loka_grouped_wgrad_workspace(ref(long))
    assert need >= 2 * 64 * 64 * 4 and wgrad(long) == wgrad(long, ws=FAKE, nws=need - 1) == WORKSPACE and wgrad(long, ws=OTHER, nws=need) == ALIGN
    assert B.lib().loka_grouped_wgrad_workspace(ref(desc())) == 0
    for x_rows in (0, MOST + 1):
        assert gemm(desc(x_rows=x_rows), index=FAKE) == linear(desc(x_rows=x_rows), index=FAKE) == SHAPE
    for form in (-1, 2):
        assert gemm(desc(w_form=form)) == linear(desc(w_form=form)) == UNSUPPORTED
    assert linear(desc(), ld=15) == SHAPE
    assert B.lib().loka_grouped_linear_workspace(ref(desc()), 0) == 0                   # (quantized inside the product)
    many = desc(rows=4096, N=1024)
    need = B.lib().loka_grouped_linear_workspace(ref(many), 0)
    assert need >= 4096 * 128 + 4096 * 4 and linear(many, ws=None, nws=0) == linear(many, nws=need - 1) == WORKSPACE and linear(many, ws=OTHER, nws=need) == ALIGN


def test_combine_refusals():
    def desc(tokens=4, cols=16, rows=8, top_k=2):
        return B.CombineDesc(tokens, cols, rows, top_k)

    def call(d, y=FAKE, slot=FAKE, weight=None, res=None, out=FAKE):
        return B.lib().loka_combine(ref(d), y, slot, weight, res, out, None)

    def back(d, dout=FAKE, y=FAKE, slot=FAKE, weight=None, dy=FAKE, dweight=FAKE):
        return B.lib().loka_combine_backward(ref(d), dout, y, slot, weight, dy, dweight, None)

    for n in ("y", "slot", "out"):
        assert call(desc(), **{n: None}) == NULL, n
    for n in ("y", "slot", "weight", "res", "out"):
        assert call(desc(), **{n: ODD}) == ALIGN, n
    assert back(desc(), dout=None) == back(desc(), slot=None) == back(desc(), y=None) == back(desc(), dy=None, dweight=None) == NULL
    for n in ("dout", "y", "slot", "weight", "dy", "dweight"):
        assert back(desc(), **{n: ODD}) == ALIGN, n
    for kw in (dict(tokens=0), dict(cols=0), dict(cols=(1 << 20) + 1), dict(rows=0), dict(rows=MOST + 1), dict(top_k=0), dict(top_k=17), dict(tokens=1 << 30),
               dict(rows=MOST, cols=1 << 20)):
        assert call(desc(**kw)) == back(desc(**kw)) == SHAPE, kw


def test_binding_looks_at_every_tensor():
    """On the host every tensor is on the wrong device; sizes and types are looked at first."""
    f, i, b, u = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(8, 16, dtype=torch.bfloat16), torch.zeros(8, 128, dtype=torch.uint8)
    off, row = torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)
    d = B.make_grouped_desc(8, 16, 16, 2)
    wq, sw, s = torch.zeros(2, 16, 128, dtype=torch.uint8), torch.zeros(2, 16), torch.zeros(8, 1)
    xt = torch.zeros(2, 16, 128, dtype=torch.uint8)
    good = [lambda: B.loka_route(f, 2), lambda: B.loka_route_backward(f, i, f[:, :2].contiguous()), lambda: B.loka_grouped_quantize(b),
            lambda: B.loka_grouped_gemm(d, u, s, wq, sw, off), lambda: B.loka_grouped_linear(d, b, wq, sw, off, index=row),
            lambda: B.loka_grouped_wgrad(d, xt, sw, xt, sw, off), lambda: B.loka_combine(b, i), lambda: B.loka_combine_backward(b[:4], b, i)]
    for call in good:
        with pytest.raises(AssertionError, match="one GPU"):
            call()
    bad = [lambda: B.loka_route(f.double(), 2), lambda: B.loka_route(f.t(), 2), lambda: B.loka_route(f[0], 2),
           lambda: B.loka_route_backward(f, i.long(), f[:, :2].contiguous()), lambda: B.loka_route_backward(f, i, f), lambda: B.loka_route_backward(f, i[:3], f[:, :2].contiguous()),
           lambda: B.loka_grouped_quantize(f), lambda: B.loka_grouped_quantize(b, offsets=off.long()), lambda: B.loka_grouped_quantize(b, index=row.long()),
           lambda: B.loka_grouped_quantize(b, along=False), lambda: B.loka_grouped_gemm(d, u[:, :64], s, wq, sw, off), lambda: B.loka_grouped_gemm(d, u[:7], s, wq, sw, off),
           lambda: B.loka_grouped_gemm(d, u, s, wq[:1], sw, off), lambda: B.loka_grouped_gemm(d, u, s, wq, sw[:1], off), lambda: B.loka_grouped_gemm(d, u, s, wq, sw, off[:2]),
           lambda: B.loka_grouped_gemm(d, u, s[:7], wq, sw, off), lambda: B.loka_grouped_gemm(d, u, s, wq, sw, off, index=row[:7]),
           lambda: B.loka_grouped_linear(d, b[:, :8], wq, sw, off), lambda: B.loka_grouped_linear(d, b[:7], wq, sw, off),
           lambda: B.loka_grouped_wgrad(d, xt, sw, xt[:, :15], sw, off), lambda: B.loka_combine(b, i.long()), lambda: B.loka_combine(b.float(), i), lambda: B.loka_combine(b, i, f),
           lambda: B.loka_combine(b, i, residual=b), lambda: B.loka_combine(b, i, out=b), lambda: B.loka_combine_backward(b, b, i), lambda: B.loka_combine_backward(b[:4], None, i)]
    for n, call in enumerate(bad):
        with pytest.raises(AssertionError) as e:
            call()
        assert "one GPU" not in str(e.value), n
    for call in (lambda: B.loka_route(torch.zeros(0, 8), 2), lambda: B.loka_route(f, 0), lambda: B.loka_route(f, 17), lambda: B.loka_route(torch.zeros(1, 1025), 2),
                 lambda: B.loka_grouped_quantize(b, groups=3), lambda: B.loka_grouped_quantize(b, groups=0), lambda: B.loka_grouped_quantize(b[:0]),
                 lambda: B.loka_grouped_quantize(b, groups=2000), lambda: B.loka_combine(b, torch.zeros(4, 17, dtype=torch.int32)), lambda: B.loka_combine(b[:0], i),
                 lambda: B.loka_grouped_gemm(B.make_grouped_desc(8, 0, 16, 2), u, s, wq, sw, off), lambda: B.loka_grouped_wgrad(B.make_grouped_desc(8, 16, 1 << 21, 2), xt, sw, xt, sw, off),
                 lambda: B.loka_grouped_linear(B.make_grouped_desc(-1, 16, 16, 2), b, wq, sw, off)):
        with pytest.raises(B.LokaError):
            call()


@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_plain_weights_gradient_against_differences(score, renorm):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(6, 9, generator=g, dtype=torch.float64)
    x[2, 3:] = -float("inf")            # three left of four
    e = X.choose(x, 4)
    assert (e[2] >= 0).sum() == 3
    c = torch.randn(6, 4, generator=g, dtype=torch.float64)
    x.requires_grad_(True)
    (X.weights(x, e, score, renorm, 1.7) * c).sum().backward()
    h = 1e-6                           # differences: error h^2, and 2^-52 / h
    with torch.no_grad():
        for t in range(6):
            for j in range(9):
                if torch.isinf(x[t, j]):
                    continue
                up, down = x.detach().clone(), x.detach().clone()
                up[t, j] += h
                down[t, j] -= h
                d = ((X.weights(up, e, score, renorm, 1.7) - X.weights(down, e, score, renorm, 1.7)) * c).sum() / (2 * h)
                assert abs(float(d - x.grad[t, j])) < 1e-8


def test_plain_combine_gradient_against_differences():
    g = torch.Generator().manual_seed(6)
    y, w, c = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((7, 5), (4, 2), (4, 5)))
    slots = torch.tensor([[0, 3], [5, 1], [-1, 2], [6, -1]])
    dy, dw = X.combine_backward(c, y, slots, w, 7)
    loss = lambda y, w: (X.combine(y, slots, w) * c).sum()
    h = 1e-6
    for m, d, f in ((y, dy, lambda v: loss(v, w)), (w, dw, lambda v: loss(y, v))):
        for i in range(m.shape[0]):
            for j in range(m.shape[1]):
                up, down = m.clone(), m.clone()
                up[i, j] += h
                down[i, j] -= h
                assert abs(float((f(up) - f(down)) / (2 * h) - d[i, j])) < 1e-8
    assert float(dw[2, 0]) == 0 and bool((dy[4] == 0).all())


def test_plain_choice_and_order():
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[1.0, 3.0, 3.0, 2.0], [-inf, -inf, 0.0, -inf], [-inf] * 4, [nan, inf, -0.0, 0.0], [0.0, -0.0, nan, nan]])
    e = X.choose(x, 3)
    assert e.tolist() == [[1, 2, 3], [2, -1, -1], [-1, -1, -1], [0, 1, 2], [2, 3, 0]]
    slots, rows, offsets = X.order(e, 4)
    assert offsets.tolist() == [0, 2, 4, 8, 10] and rows.tolist() == [3, 4, 0, 3, 0, 1, 3, 4, 0, 4, -1, -1, -1, -1, -1]
    assert slots.tolist() == [[2, 4, 8], [5, -1, -1], [-1, -1, -1], [0, 3, 6], [7, 9, 1]]
