"""The residual norm with a small eps over all of bf16's range: rows whose squares fp32 does not hold, too large or too small, in every
layout of the lanes, against plain 64-bit forms."""
import pytest
import torch

import plain_ops as P
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MODES = {"row": B.SCALE_ROW, "block": B.SCALE_BLOCK_1x128, "pow2": B.SCALE_BLOCK_1x128_POW2}
# fp32 roundings, relative: at most 32 squares in a thread, 6 exchanges and 16 waves, the square and h themselves (rstd has half of all
# that); then division, root, mean, and the products with rstd, gamma and a scale's factors.  A power of two in front adds none.
REL = ((32 + 6 + 16 + 3) / 2 + 10) * P.F32
COLS = [16, 128, 256, 512, 1008, 2048, 4096, 8192, 16384, 32768]
EXPONENTS = [-132, -126, -110, -96, -75, -63, -50, -46, -44, -40, -20, 0, 20, 45, 49, 51, 55, 62, 64, 75, 90, 110, 120]


def _rows(cols, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(len(EXPONENTS), cols, device=DEV, generator=g)
    unit = P.pow2(torch.tensor(EXPONENTS, device=DEV))[:, None]
    return (x.bfloat16().double() * unit).to(torch.bfloat16), (1 + 0.2 * torch.randn(cols, device=DEV, generator=g)).bfloat16()


@pytest.mark.parametrize("eps", [0.0, 1e-42, 1e-30])
@pytest.mark.parametrize("cols", COLS)
def test_bf16_and_mxfp4_output(cols, eps):
    x, w = _rows(cols, cols)
    eps = float(torch.tensor(eps))     # (as the call takes it)
    _, rstd, y = P.rms_forward(x, None, w, eps)
    got = B.loka_add_rmsnorm(x, None, w, eps, out=B.RMS_OUT_BF16, want_rstd=True)
    # where a product is subnormal it is rounded to multiples of 2^-149: h gamma (then times rstd), and y; bf16's are multiples of 2^-133
    low = 2.0 ** -150 * (1 + rstd.clamp_max(2.0 ** 45))      # (rows with a larger rstd are scaled up first)
    assert bool(((got.y.double() - y).abs() <= (2.0 ** -8 + REL) * y.abs() + low + 2.0 ** -134).all())
    held = rstd.view(-1) < 2.0 ** 127.9
    err = (got.rstd.double() - rstd.view(-1)).abs()
    assert bool((err <= REL * rstd.view(-1) + 2.0 ** -150)[held].all())
    got = B.loka_add_rmsnorm(x, None, w, eps, out=B.RMS_OUT_MXFP4)
    g = torch.zeros(len(EXPONENTS), P.padded(cols), dtype=torch.float64, device=DEV)
    g[:, :cols] = y
    g = g.view(len(EXPONENTS), -1, 32)
    amax, byte = g.abs().amax(-1), got.scales.long()
    lo, hi = (torch.where(amax > 0, P.exponent((amax * f).clamp_min(1e-300)) - 2, -127).clamp_min(-127) + 127 for f in (1 - REL, 1 + REL))
    assert bool(((byte >= lo) & (byte <= hi)).all())
    unit = P.pow2(byte - 127)[..., None]
    t, v = g / unit, P.mx_values(got.y, got.scales).view_as(g) / unit
    step = torch.where(t.abs() < 2, 0.5, torch.where(t.abs() < 4, 1.0, 2.0))
    assert bool(((v - t.clamp(-6, 6)).abs() <= step / 2 + 2 * REL * t.abs() + low[..., None] / unit).all())


@pytest.mark.parametrize("eps", [0.0, 1e-30])
@pytest.mark.parametrize("cols,mode", [(c, m) for c in COLS for m in MODES if m == "row" or c % 128 == 0])
def test_e4m3_output_and_checkpoint(cols, mode, eps):
    x, w = _rows(cols, 3 * cols)
    got = B.loka_add_rmsnorm(x, None, w, eps, out_mode=MODES[mode], ckpt_mode=MODES[mode])
    # the checkpoint is loka_quantize's, to the bit, whatever the norm does with the row
    q, s = B.loka_quantize(x, MODES[mode])
    assert torch.equal(got.hq, q) and torch.equal(got.hs.view(-1), s)
    _, _, y = P.rms_forward(x, None, w, float(torch.tensor(eps)))
    g = y.view(len(EXPONENTS), 1 if mode == "row" else cols // 128, -1)
    amax, scale = g.abs().amax(-1).clamp_min(1e-12), got.scales.double().view(len(EXPONENTS), -1)
    if mode == "pow2":
        assert torch.equal(scale, P.pow2(P.exponent(scale)))
        assert bool((amax / scale <= 448 * (1 + REL)).all()) and bool((2 * amax / scale > 448 * (1 - REL)).all())
    else:
        assert bool(((scale - amax / 448).abs() <= REL * amax / 448).all())
    t = (g / scale[..., None]).view(y.shape)
    err = (P.e4m3_values(got.y).view(y.shape) - t.clamp(-448, 448)).abs()
    assert bool((err <= P.e4m3_step(t) / 2 + 2 * REL * t.abs()).all())


@pytest.mark.parametrize("cols", COLS)
def test_neighbours_of_such_rows_and_values_that_are_not_finite(cols):
    # rows that are scaled share waves with rows that are not: each as it is alone
    x, w = _rows(cols, 5 * cols)
    x[3, 1], x[7, cols - 1], x[11] = float("nan"), float("inf"), 0
    for out in (B.RMS_OUT_BF16, B.RMS_OUT_E4M3, B.RMS_OUT_MXFP4):
        for eps in (0.0, 1e-30):
            all_rows = B.loka_add_rmsnorm(x, x, w, eps, out=out, ckpt_mode=B.SCALE_ROW)
            for i in range(len(EXPONENTS)):
                alone = B.loka_add_rmsnorm(x[i:i + 1], x[i:i + 1], w, eps, out=out, ckpt_mode=B.SCALE_ROW)
                for a, b in zip(all_rows, alone):
                    if a is not None:
                        a, b = a[i:i + 1].float(), b.float()
                        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)), (out, eps, i)
    got = B.loka_add_rmsnorm(x, None, w, 0.0, out=B.RMS_OUT_BF16)
    _, _, y = P.rms_forward(x, None, w, 0.0)
    assert torch.equal(torch.isnan(got.y), torch.isnan(y))


@pytest.mark.parametrize("exponent", [-40, -35, 50, 60])
def test_backward_from_such_rows(exponent):
    # (an 8-bit checkpoint holds rows above its floor of 1e-12 and all larger ones)
    rows, cols = 40, 1024
    g = torch.Generator(device=DEV).manual_seed(exponent + 100)
    x = (torch.randn(rows, cols, device=DEV, generator=g) * 2.0 ** exponent).bfloat16()
    dy, w = torch.randn(rows, cols, device=DEV, generator=g).bfloat16(), (1 + 0.2 * torch.randn(cols, device=DEV, generator=g)).bfloat16()
    f = B.loka_add_rmsnorm(x, None, w, 0.0, out=B.RMS_OUT_BF16, ckpt_mode=B.SCALE_ROW)
    dx, dg = B.loka_rmsnorm_backward(dy, f.hq, f.hs, f.rstd, w, ckpt_mode=B.SCALE_ROW)
    h = P.e4m3_values(f.hq) * f.hs.double()[:, None]
    want, wdg, mag, dmag = P.rms_backward(dy, h, f.rstd.double()[:, None], w, None)
    # the inner sum: 32 terms in a thread, 6 exchanges, 16 waves; 4 roundings a term and 4 on the way out
    assert bool(((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + (32 + 6 + 16 + 8) * P.F32 * 2 * mag).all())
    assert bool(((dg.double() - wdg).abs() <= (rows + 512 + 8) * P.F32 * dmag).all())


@pytest.mark.parametrize("eps", [1e-27, 1e-12, 1e-5])
@pytest.mark.parametrize("cols", COLS)
def test_small_rows_beside_a_larger_eps(cols, eps):
    # sums that vanish beside eps, down to nothing; up to where fp32 holds the squares
    x, w = _rows(cols, cols)
    x = x[:EXPONENTS.index(45) + 1]
    eps = float(torch.tensor(eps))
    _, rstd, y = P.rms_forward(x, None, w, eps)
    got = B.loka_add_rmsnorm(x, None, w, eps, out=B.RMS_OUT_BF16, want_rstd=True)
    low = 2.0 ** -150 * (1 + rstd)
    assert bool(((got.y.double() - y).abs() <= (2.0 ** -8 + REL) * y.abs() + low + 2.0 ** -134).all())
    assert bool(((got.rstd.double() - rstd.view(-1)).abs() <= REL * rstd.view(-1)).all())
