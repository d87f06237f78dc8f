"""The residual norm and its backward pass within bounds counted from the kernels' own roundings: at most 32 elements of a row in a thread,
6 exchanges in a wave, 16 waves."""
import pytest
import torch

import plain_ops as P
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = [(1, 4096), (40, 128), (64, 256), (33, 512), (9, 1008), (130, 1024), (40, 2048), (300, 4096), (7, 4112), (30, 8192), (5, 16384), (6, 16400), (3, 32768),
          (4000, 1280), (2049, 4096)]


def _inputs(rows, cols):
    g = torch.Generator(device=DEV).manual_seed(rows * 7 + cols)
    x, r = (torch.randn(rows, cols, device=DEV, generator=g) for _ in range(2))
    x[:, ::97] *= 50.0
    return x.bfloat16(), r.bfloat16(), (1 + 0.2 * torch.randn(cols, device=DEV, generator=g)).bfloat16(), g


@pytest.mark.parametrize("mode", ["row", "block"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_codes_are_rounded_once(rows, cols, mode):
    if mode == "block" and cols % 128:
        pytest.skip("blocks of 128")
    x, r, w, _ = _inputs(rows, cols)
    m = B.SCALE_ROW if mode == "row" else B.SCALE_BLOCK_1x128
    got = B.loka_add_rmsnorm(x, r, w, 1e-5, out_mode=m, ckpt_mode=m)
    h = (x.float() + r.float()).double()            # (the sum is defined in fp32)
    # code = e4m3((h gamma) * (448 / max|h gamma|)), each product and the quotient rounded, and the maximum is one of the products; rstd is in
    # neither.  The checkpoint: 448 / max|h| and its product with h
    for codes, v, roundings in ((got.y, h * w.double(), 4), (got.hq, h, 2)):
        t = v.view(rows, -1, cols if mode == "row" else 128)
        t = (t * (448 / t.abs().amax(-1, keepdim=True))).view(rows, cols)
        err = (P.e4m3_values(codes).view(rows, cols) - t).abs()
        tol = P.e4m3_step(t) / 2 + (roundings + 1e-6) * P.F32 * t.abs()
        assert bool((err <= tol).all()), float((err - P.e4m3_step(t) / 2).max())


@pytest.mark.parametrize("gamma,dh", [(True, True), (False, False)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_norm_and_gradient(rows, cols, gamma, dh):
    x, r, w, g = _inputs(rows, cols)
    w = w if gamma else None
    f = B.loka_add_rmsnorm(x, r, w, 1e-5, out=B.RMS_OUT_BF16, ckpt_mode=B.SCALE_ROW)
    h, rstd, y = P.rms_forward(x.float() + r.float(), None, w, 1e-5)
    # squares and sums (rstd has half of their error), division, addition of eps, root and its quotient; then two products
    stat = ((1 + 32 + 6 + 16) / 2 + 4) * P.F32
    assert bool(((f.rstd.double() - rstd.view(-1)).abs() <= stat * rstd.view(-1)).all())
    assert bool(((f.y.double() - y).abs() <= (2.0 ** -8 + stat + 2 * P.F32) * y.abs()).all())
    dy = torch.randn(rows, cols, device=DEV, generator=g).bfloat16()
    e = torch.randn(rows, cols, device=DEV, generator=g).bfloat16() if dh else None
    dx, dg = B.loka_rmsnorm_backward(dy, f.hq, f.hs, f.rstd, w, e, ckpt_mode=B.SCALE_ROW)
    hc = P.e4m3_values(f.hq) * f.hs.double()[:, None]
    want, wdg, mag, dmag = P.rms_backward(dy, hc, f.rstd.double()[:, None], w, e)
    # n = code * (scale * rstd): 2 roundings; a term of the mean: 2 + 1, then the sum and the division; dx: n, its product with the mean and two
    # sums' roundings
    inner = (2 + 1 + 32 + 6 + 16 + 1) * P.F32
    assert bool(((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + (inner + 6 * P.F32) * mag).all())
    assert bool(((dg.double() - wdg).abs() <= (2 + rows + 512) * P.F32 * dmag).all())
