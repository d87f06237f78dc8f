"""Plain 64-bit forms of the MXFP4 and residual-norm operators, for the tests (test infrastructure, torch only).

Nothing here calls the library.  Roundings are counted in half steps: bf16 2^-8, fp32 2^-24, e4m3 2^-4 of the value."""
from __future__ import annotations

import torch

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
F32 = 2.0 ** -24        # half a step of binary32, relative


def padded(k: int) -> int:
    return (k + 127) // 128 * 128


def exponent(v: torch.Tensor) -> torch.Tensor:
    """floor(log2 v) of positive fp64 values (normal in binary64: every bf16 and fp32 is)."""
    return (v.contiguous().view(torch.int64) >> 52) - 1023


def pow2(e: torch.Tensor) -> torch.Tensor:
    """2^e of integers, exactly (torch.pow is not on every device)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def e2m1_codes(t: torch.Tensor) -> torch.Tensor:
    """Magnitude codes 0 .. 7 of |t|: to nearest, ties to the even code, above 6 to 6."""
    a = t.abs()
    c = torch.zeros_like(a, dtype=torch.int64)
    for i in range(7):
        mid = (E2M1[i] + E2M1[i + 1]) / 2
        c += (a > mid) if i % 2 == 0 else (a >= mid)
    return c


def mx_quantize(x: torch.Tensor):
    """[rows, cols] (any type) -> (packed codes uint8 [rows, Kp / 2], scale bytes uint8 [rows, Kp / 32])."""
    rows, cols = x.shape
    g = torch.zeros(rows, padded(cols), dtype=torch.float64, device=x.device)
    g[:, :cols] = x.double()
    g = g.view(rows, -1, 32)
    amax = g.abs().amax(-1)                                       # (a NaN is the largest)
    bad = ~torch.isfinite(amax)
    byte = torch.where(amax > 0, exponent(torch.where(bad, 1.0, amax).clamp_min(1e-300)) - 2, -127).clamp_min(-127) + 127
    code = e2m1_codes(g * pow2(127 - byte)[..., None]) | (torch.signbit(g).long() << 3)
    code = torch.where(bad[..., None], 0, code).view(rows, -1, 2)
    return (code[..., 0] | code[..., 1] << 4).to(torch.uint8), torch.where(bad, 255, byte).to(torch.uint8)


def mx_values(q: torch.Tensor, s: torch.Tensor) -> torch.Tensor:
    """fp64 [rows, Kp] of stored codes."""
    q = q.long()
    code = torch.stack((q & 15, q >> 4), -1).view(q.shape[0], -1)
    v = torch.tensor(E2M1, dtype=torch.float64, device=q.device)[code & 7] * (1 - 2 * (code >> 3)).double()
    scale = torch.where(s == 255, torch.nan, pow2(s.long() - 127))
    return v * scale.repeat_interleave(32, 1)


def e4m3_values(q: torch.Tensor) -> torch.Tensor:
    return q.view(torch.float8_e4m3fn).double()


def e4m3_step(t: torch.Tensor) -> torch.Tensor:
    """Spacing of e4m3 values around t."""
    return pow2(exponent(t.abs().clamp_min(2.0 ** -6)) - 3)


def rms_forward(x, residual, gamma, eps):
    """(h, rstd [rows, 1], y) in fp64."""
    h = x.double() if residual is None else x.double() + residual.double()
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, rstd, h * rstd * (1.0 if gamma is None else gamma.double())


def rms_backward(dy, h, rstd, gamma, dh):
    """(dx, dgamma, and the magnitudes that went into each, for error bounds) in fp64; h: the checkpoint's values."""
    n = h * rstd
    g = dy.double() * (1.0 if gamma is None else gamma.double())
    c = (g * n).mean(1, keepdim=True)
    dx = rstd * (g - n * c) + (0 if dh is None else dh.double())
    mag = rstd * (g.abs() + n.abs() * (g * n).abs().mean(1, keepdim=True)) + (0 if dh is None else dh.double().abs())
    return dx, (dy.double() * n).sum(0), mag, (dy.double() * n).abs().sum(0)
