"""What the MXFP4 and residual-norm entry points refuse, before any HIP call (no GPU), and the plain forms that the GPU tests
compare with, against differences."""
import ctypes

import pytest
import torch

import plain_ops as P
from paper_2605_10886_amd import binding as B

FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
BF = torch.bfloat16


def test_quantize_and_dequantize():
    q = B.lib().loka_mxfp4_quantize
    assert q(None, 1, 1, 1, 0, FAKE, FAKE, None) == q(FAKE, 1, 1, 1, 0, None, FAKE, None) == q(FAKE, 1, 1, 1, 0, FAKE, None, None) == B.LOKA_ERR_NULL
    for rows, cols, ld in ((0, 8, 8), (8, 0, 8), (8, 8, 7), (1 << 31, 8, 8), (8, 1 << 31, 1 << 31), (-1, 8, 8)):
        assert q(FAKE, rows, cols, ld, 0, FAKE, FAKE, None) == B.LOKA_ERR_SHAPE
    assert q(ODD, 8, 8, 8, 0, FAKE, FAKE, None) == q(FAKE, 8, 8, 8, 0, ODD, FAKE, None) == q(FAKE, 8, 8, 8, 0, FAKE, ODD, None) == B.LOKA_ERR_ALIGN
    d = B.lib().loka_mxfp4_dequantize
    assert d(None, FAKE, 8, 8, FAKE, 8, None) == d(FAKE, None, 8, 8, FAKE, 8, None) == d(FAKE, FAKE, 8, 8, None, 8, None) == B.LOKA_ERR_NULL
    assert d(FAKE, FAKE, 0, 8, FAKE, 8, None) == d(FAKE, FAKE, 8, 8, FAKE, 7, None) == B.LOKA_ERR_SHAPE
    assert d(ODD, FAKE, 8, 8, FAKE, 8, None) == d(FAKE, FAKE, 8, 8, ODD, 8, None) == B.LOKA_ERR_ALIGN
    assert [B.loka_mxfp4_padded(k) for k in (-1, 0, 1, 128, 129, (1 << 63) - 1)] == [-1, -1, 128, 128, 256, -1]


def _gemm(d, xq=FAKE, sx=FAKE, wq=FAKE, sw=FAKE, out=FAKE, y=None, ws=None, nws=0):
    return B.lib().loka_mxfp4_gemm(ctypes.byref(d), xq, sx, wq, sw, out, y, ws, nws, None)


def _linear(d, x=FAKE, ld=64, wq=FAKE, sw=FAKE, out=FAKE, y=None, ws=None, nws=0):
    return B.lib().loka_mxfp4_linear(ctypes.byref(d), x, ld, wq, sw, out, y, ws, nws, None)


def test_products():
    good = B.make_mxfp4_desc(64, 48, 64)
    for name in ("xq", "sx", "wq", "sw", "out"):
        assert _gemm(good, **{name: None}) == B.LOKA_ERR_NULL
        assert _gemm(good, **{name: ODD}) == B.LOKA_ERR_ALIGN
    assert _gemm(good, y=ODD) == _gemm(good, ws=ODD, nws=64) == B.LOKA_ERR_ALIGN
    for name in ("M", "N", "K", "batch"):
        for v in (0, -1, 1 << 31):
            d = B.make_mxfp4_desc(64, 48, 64)
            setattr(d, name, v)
            assert _gemm(d) == B.LOKA_ERR_SHAPE
            assert _linear(d, ld=1 << 32) == B.LOKA_ERR_SHAPE
            assert B.lib().loka_mxfp4_gemm_workspace(ctypes.byref(d)) == 0 == B.lib().loka_mxfp4_linear_workspace(ctypes.byref(d))
    for name, v in (("norm", B.NORM_RMSNORM), ("act", B.ACT_HARDSWISH), ("variant", 0)):
        d = B.make_mxfp4_desc(64, 48, 64)
        setattr(d, name, v)
        assert _gemm(d) == _linear(d) == B.LOKA_ERR_UNSUPPORTED
    for name, v, st in (("strideX", 64 * 127, B.LOKA_ERR_SHAPE), ("strideX", -128, B.LOKA_ERR_SHAPE), ("strideW", 48 * 128 - 128, B.LOKA_ERR_SHAPE),
                        ("strideO", 64 * 48 - 1, B.LOKA_ERR_SHAPE), ("strideX", 64 * 128 + 64, B.LOKA_ERR_ALIGN), ("strideW", 48 * 128 + 1, B.LOKA_ERR_ALIGN)):
        d = B.make_mxfp4_desc(64, 48, 64, 3)
        setattr(d, name, v)
        assert _gemm(d) == st, (name, v)
    for name in ("x", "wq", "sw", "out"):
        assert _linear(good, **{name: None}) == B.LOKA_ERR_NULL
        assert _linear(good, **{name: ODD}) == B.LOKA_ERR_ALIGN
    assert _linear(good, ld=63) == B.LOKA_ERR_SHAPE
    assert _linear(B.make_mxfp4_desc(64, 48, 64, 2)) == B.LOKA_ERR_UNSUPPORTED
    assert _linear(good) == _linear(good, ws=FAKE, nws=8) == B.LOKA_ERR_WORKSPACE
    need = B.lib().loka_mxfp4_linear_workspace(ctypes.byref(good))
    assert need >= 64 * 128 // 2 + 64 * 4 and _linear(good, ws=ctypes.c_void_p(0x1008), nws=need) == B.LOKA_ERR_ALIGN
    assert B.lib().loka_mxfp4_linear_workspace(ctypes.byref(B.make_mxfp4_desc(16, 48, 64))) == 0


def _rms(d, x=FAKE, res=None, gamma=None, h=None, y=FAKE, s=FAKE, hq=None, hs=None, rstd=None):
    return B.lib().loka_add_rmsnorm(ctypes.byref(d), x, res, gamma, h, y, s, hq, hs, rstd, None)


def _back(d, dy=FAKE, hq=FAKE, hs=FAKE, rstd=FAKE, gamma=None, dh=None, dx=FAKE, dg=None, ws=None, nws=0):
    return B.lib().loka_rmsnorm_backward(ctypes.byref(d), dy, hq, hs, rstd, gamma, dh, dx, dg, ws, nws, None)


def test_residual_norm():
    def desc(rows=8, cols=256, ld_x=256, ld_r=256, out=B.RMS_OUT_E4M3, out_mode=B.SCALE_ROW, ckpt_mode=B.SCALE_BLOCK_1x128, eps=1e-5):
        return B.RmsDesc(rows, cols, ld_x, ld_r, out, out_mode, ckpt_mode, eps)

    assert _rms(desc(), x=None) == _rms(desc(), y=None) == _rms(desc(), s=None) == _rms(desc(), hq=FAKE) == _rms(desc(), hs=FAKE) == B.LOKA_ERR_NULL
    for kw in (dict(rows=0), dict(rows=-4), dict(rows=1 << 31), dict(cols=0), dict(cols=120), dict(cols=32784, ld_x=32784), dict(ld_x=248)):
        assert _rms(desc(**kw)) == B.LOKA_ERR_SHAPE, kw
        assert _back(desc(**kw)) == B.LOKA_ERR_SHAPE, kw
    assert _rms(desc(ld_r=248), res=FAKE) == _back(desc(ld_r=248), dh=FAKE) == B.LOKA_ERR_SHAPE
    assert _rms(desc(ld_x=260)) == _back(desc(ld_x=260)) == _rms(desc(ld_r=260), res=FAKE) == _back(desc(ld_r=260), dh=FAKE) == B.LOKA_ERR_ALIGN
    assert _rms(desc(cols=208, out_mode=B.SCALE_BLOCK_1x128)) == _rms(desc(cols=208), hq=FAKE, hs=FAKE) == _back(desc(cols=208)) == B.LOKA_ERR_SHAPE
    for mode in (B.SCALE_TENSOR, B.SCALE_COL, B.SCALE_BLOCK_128x128, B.SCALE_BLOCK_128x1, 8, -1):
        assert _rms(desc(out_mode=mode)) == _rms(desc(ckpt_mode=mode), hq=FAKE, hs=FAKE) == _back(desc(ckpt_mode=mode)) == B.LOKA_ERR_UNSUPPORTED
    for kw in (dict(out=3), dict(out=-1), dict(eps=-1.0), dict(eps=float("nan"))):
        assert _rms(desc(**kw)) == B.LOKA_ERR_UNSUPPORTED
    for name in ("x", "res", "gamma", "h", "y", "s", "rstd"):
        assert _rms(desc(), **{name: ODD}) == B.LOKA_ERR_ALIGN, name
    assert _rms(desc(), hq=ODD, hs=FAKE) == _rms(desc(), hq=FAKE, hs=ODD) == B.LOKA_ERR_ALIGN
    for name in ("dy", "hq", "hs", "rstd", "dx"):
        assert _back(desc(), **{name: None}) == B.LOKA_ERR_NULL, name
    for name in ("dy", "hq", "hs", "rstd", "dx", "gamma", "dh", "dg"):
        assert _back(desc(), **{name: ODD}) == B.LOKA_ERR_ALIGN, name
    OTHER = ctypes.c_void_p(0x2000)        # an output over an input that has another row stride
    assert _rms(desc(ld_x=264), h=FAKE) == _rms(desc(ld_r=264), x=OTHER, res=FAKE, h=FAKE) == B.LOKA_ERR_SHAPE
    assert _back(desc(ld_x=264)) == _back(desc(ld_r=264), dy=OTHER, dh=FAKE) == B.LOKA_ERR_SHAPE
    assert _back(desc(), dg=FAKE) == _back(desc(), dg=FAKE, ws=FAKE, nws=16) == B.LOKA_ERR_WORKSPACE
    need = B.lib().loka_rmsnorm_backward_workspace(ctypes.byref(desc()))
    assert need >= 256 * 4 and _back(desc(), dg=FAKE, ws=ctypes.c_void_p(0x1008), nws=need) == B.LOKA_ERR_ALIGN
    assert B.lib().loka_rmsnorm_backward_workspace(ctypes.byref(desc(cols=0))) == 0


def test_binding_looks_at_every_tensor():
    x = torch.zeros(8, 64, dtype=BF)
    for bad in (torch.zeros(8, 64), x[0], x.t()):
        with pytest.raises(AssertionError):
            B.loka_mxfp4_quantize(bad)
        with pytest.raises(AssertionError):
            B.loka_add_rmsnorm(bad)
    with pytest.raises(AssertionError):
        B.loka_mxfp4_quantize(x)                                                  # not on the GPU
    with pytest.raises(AssertionError):
        B.loka_add_rmsnorm(x)
    for rows, cols in ((0, 64), (8, 0)):
        for call in (B.loka_mxfp4_quantize, B.loka_add_rmsnorm):
            with pytest.raises(B.LokaError) as e:
                call(torch.zeros(rows, cols, dtype=BF))
            assert e.value.status == B.LOKA_ERR_SHAPE
    q, s = torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8)
    for args in ((q, s[:7], 64), (q, s, 129), (q.float(), s, 64), (q, s.t(), 64)):
        with pytest.raises(AssertionError):
            B.loka_mxfp4_dequantize(*args)
    d = B.make_mxfp4_desc(8, 8, 64)
    for i in range(4):
        ops = [q, s, q, s]
        ops[i] = ops[i][:7]
        with pytest.raises(AssertionError):
            B.loka_mxfp4_gemm(d, *ops)
    with pytest.raises(AssertionError):
        B.loka_mxfp4_gemm(B.make_mxfp4_desc(8, 8, 64, 2), q, s, q, s)             # operands of one problem
    with pytest.raises(AssertionError):
        B.loka_mxfp4_linear(d, x[:7], q, s)
    with pytest.raises(AssertionError):
        B.loka_mxfp4_linear(d, x, q[:7], s)
    with pytest.raises(B.LokaError):
        B.loka_mxfp4_gemm(B.make_mxfp4_desc(0, 8, 64), q, s, q, s)
    for kw in (dict(residual=x[:7]), dict(gamma=torch.zeros(63, dtype=BF)), dict(gamma=torch.zeros(64))):
        with pytest.raises(AssertionError):
            B.loka_add_rmsnorm(x, **kw)
    with pytest.raises(B.LokaError):
        B.loka_add_rmsnorm(x, out_mode=B.SCALE_BLOCK_1x128)                       # 64 columns
    hq, hs, rstd = torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8), torch.zeros(8)
    for args in ((x, hq[:7], hs, rstd), (x, hq, hs[:7], rstd), (x, hq, hs, rstd[:7]), (x, hq, hs, rstd, torch.zeros(63, dtype=BF)),
                 (x, hq, hs, rstd, None, x[:7]), (x, hq, hs, rstd)):
        with pytest.raises(AssertionError):
            B.loka_rmsnorm_backward(*args, ckpt_mode=B.SCALE_ROW)


def test_plain_quantizer_on_known_groups():
    x = torch.zeros(3, 64)
    x[0, :8] = torch.tensor([0.0, 0.25, 0.75, -1.25, 2.5, 5.0, 6.9, -7.9])      # amax 7.9: scale 1
    x[0, 32] = 2.0 ** -140                                                         # far below the smallest scale
    x[1, 0] = float("nan")
    x[2, 63] = -(2.0 ** 100)
    q, s = P.mx_quantize(x)
    assert s[:, :2].tolist() == [[127, 0], [255, 0], [0, 225]] and s[:, 2:].sum() == 0
    assert P.mx_values(q, s)[0, :8].tolist() == [0.0, 0.0, 1.0, -1.0, 2.0, 4.0, 6.0, -6.0]
    assert P.mx_values(q, s)[2, 63] == -(2.0 ** 100) and bool(torch.isnan(P.mx_values(q, s)[1, :32]).all())
    v = P.mx_values(*P.mx_quantize(torch.randn(50, 200, generator=torch.Generator().manual_seed(1))))
    assert torch.equal(P.mx_values(*P.mx_quantize(v)), v)                          # values of the format stay


def test_plain_gradient_against_differences():
    g = torch.Generator().manual_seed(3)
    x, up, v, dh = (torch.randn(5, 64, generator=g).double() for _ in range(4))
    w, u = (torch.randn(64, generator=g).double() for _ in range(2))
    h, rstd, _ = P.rms_forward(x, None, w, 1e-5)
    dx, dg, _, _ = P.rms_backward(up, h, rstd, w, dh)
    loss = lambda xx, ww: (up * P.rms_forward(xx, None, ww, 1e-5)[2]).sum() + (dh * xx).sum()
    t = 1e-5
    assert abs((loss(x + t * v, w) - loss(x - t * v, w)) / (2 * t) - (dx * v).sum()) < 1e-7
    assert abs((loss(x, w + t * u) - loss(x, w - t * u)) / (2 * t) - (dg * u).sum()) < 1e-7
