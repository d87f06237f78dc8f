"""The operators of a low-precision layer beside the FP8 GEMMs, as cases that can be timed and compared.

A case is one pass through the Python binding, the way a trainer or a serving loop calls it:

  requant  loka_mxfp4_quantize (plain or transposing) and loka_mxfp4_dequantize: a matrix to 4-bit codes with a scale
           per 32 elements, and the values that the codes stand for
  linear   a layer with kept 4-bit weights on bf16 activations: loka_mxfp4_linear, or, for grouped problems,
           loka_mxfp4_quantize and loka_mxfp4_gemm
  train    one training step of a 4-bit layer: forward, dX = dY W^T, dW = X^T dY, every operand quantized in the step
  norm     loka_add_rmsnorm: residual addition, RMSNorm, 8-bit codes with scales for the next layer, and (training) the
           8-bit checkpoint of the residual stream that the backward pass reads
  back     loka_rmsnorm_backward on that checkpoint

Activations are N(0, 1), Student-t(4) / sqrt 2 (heavy tails) or N(0, 1) with four channels x 100 (outliers), weights
N(0, 1/K), output gradients N(0, 0.02^2); all drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False
EPS = 1e-5
GROUP, PAD = 32, 128                # elements that share a scale; what a stored row's length is a multiple of
DEV = "cuda"

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _requant(M, K, transpose=False, dist="normal", **name):
    return dict(name, op="requant", M=M, K=K, transpose=transpose, dist=dist)


def _linear(M, K, N, batch=1, dist="normal", **name):
    return dict(name, op="linear", M=M, K=K, N=N, batch=batch, dist=dist)


def _train(M, K, N, dist="normal", **name):
    return dict(name, op="train", M=M, K=K, N=N, dist=dist)


def _norm(M, K, out="row", residual=True, ckpt=False, dist="normal", **name):
    return dict(name, op="norm", M=M, K=K, out=out, residual=residual, ckpt=ckpt, dist=dist)


def _back(M, K, ckpt="block", dh=True, dist="normal", **name):
    return dict(name, op="back", M=M, K=K, ckpt=ckpt, dh=dh, dist=dist)


def listed():
    return [
        # a large layer input measured for 4 bits: what the format does to its values
        _requant(8192, 4096, dist="student_t4", name="requant_8192x4096"),
        # the weight gradient's operand, whose contraction runs over a ragged number of rows, with outlier channels
        _requant(5013, 1008, transpose=True, dist="normal_outlier4", name="requant_t_5013x1008"),
        # one token through a square layer: latency and weight traffic
        _linear(1, 4096, 4096, name="linear_1x4096x4096"),
        # a small batch of tokens through a widening layer: weight traffic
        _linear(13, 4096, 16384, dist="normal_outlier4", name="linear_13x4096x16384"),
        # feature widths and row counts as they come
        _linear(5013, 1008, 720, dist="student_t4", name="linear_5013x1008x720"),
        # the large layer that the benchmark's headline is quoted on
        _linear(32768, 4096, 4096, dist="normal_outlier4", name="linear_32768x4096x4096"),
        # a training step of the narrowest layer of the throughput study, at its batch of 2048
        _train(2048, 256, 768, name="train_2048x256x768"),
        # a training step of a mid-sized layer
        _train(16384, 1024, 4096, dist="student_t4", name="train_16384x1024x4096"),
        # one token's norm between two layers: latency
        _norm(1, 4096, name="norm_1x4096"),
        # the norm of a large training batch: codes in row scales, and the checkpoint
        _norm(32768, 4096, ckpt=True, dist="normal_outlier4", name="norm_32768x4096_ckpt"),
        # backward passes: ragged rows and a narrow stream without a residual gradient, and a large training batch
        _back(5013, 1008, ckpt="row", dh=False, dist="student_t4", name="back_5013x1008"),
        _back(32768, 4096, dist="normal_outlier4", name="back_32768x4096"),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step)


def draw(rng):
    dist = rng.choice(("normal", "student_t4", "normal_outlier4"))
    op = rng.choice(("requant", "linear", "linear", "train", "norm", "back"))
    if op == "requant":
        M = _log(rng, 1, 16384)
        K = _log(rng, 8, min(8192, 8192 * 4096 // M))
        return _requant(M, K, transpose=rng.random() < 0.5, dist=dist)
    if op == "linear":
        if rng.random() < 0.25:         # grouped small layers
            return _linear(_log(rng, 16, 2048), _log(rng, 64, 512), _log(rng, 64, 512), batch=rng.randint(2, 32), dist=dist)
        M = _log(rng, 1, 32) if rng.random() < 0.5 else _log(rng, 33, 16384)
        return _linear(M, _log(rng, 64, 8192), _log(rng, 64, 8192), dist=dist)
    if op == "train":
        return _train(_log(rng, 64, 16384), _log(rng, 64, 2048), _log(rng, 64, 2048), dist=dist)
    M = _log(rng, 1, 32768)
    K = _log(rng, 128, min(16384, 32768 * 4096 // M), 16)
    if op == "norm":
        out = rng.choice(("row", "block", "block_pow2", "bf16"))
        if out.startswith("block"):
            K = max(128, K // 128 * 128)
        return _norm(M, K, out=out, residual=rng.random() < 0.8, ckpt=K % 128 == 0 and rng.random() < 0.6, dist=dist)
    ckpt = rng.choice(("row", "block"))
    if ckpt == "block":
        K = max(128, K // 128 * 128)
    return _back(M, K, ckpt=ckpt, dh=rng.random() < 0.7, dist=dist)


# ---- inputs

def _values(rows, cols, dist, gen):
    x = torch.randn(rows, cols, device=DEV, generator=gen)
    if dist == "student_t4":            # t(4) = z / sqrt(chi2(4) / 4), chi2(4) = -2 log(u v)
        for part in x.split(max(1, (1 << 24) // cols)):
            u = torch.rand(2, *part.shape, device=DEV, generator=gen).clamp_min_(1e-30)
            part.mul_((-0.5 * u.log().sum(0)).clamp_min_(1e-6).rsqrt_()).mul_(math.sqrt(0.5))
    elif dist == "normal_outlier4":
        x[:, torch.arange(4, device=DEV) * (cols // 4)] *= 100.0
    return x.bfloat16()


def _padded(k):
    return -(-k // PAD) * PAD


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    M, K, op = case["M"], case["K"], case["op"]
    s = dict(case)
    s["x"] = _values(M * case.get("batch", 1), K, case["dist"], gen)
    if op == "linear":                  # weights [N, K], contraction along the row, kept as codes and scales
        w = (torch.randn(case["batch"] * case["N"], K, device=DEV, generator=gen) / math.sqrt(K)).bfloat16()
        s["wq"], s["sw"] = _pack(*_mx(w.float()))
    elif op == "train":
        s["w"] = (torch.randn(K, case["N"], device=DEV, generator=gen) / math.sqrt(K)).bfloat16()
        s["dy"] = (torch.randn(M, case["N"], device=DEV, generator=gen) * 0.02).bfloat16()
    elif op in ("norm", "back"):
        s["gamma"] = (1 + 0.1 * torch.randn(K, device=DEV, generator=gen)).bfloat16()
        s["res"] = _values(M, K, "normal", gen) if case.get("residual") else None
        if op == "back":
            s["dy"] = (torch.randn(M, K, device=DEV, generator=gen) * 0.02).bfloat16()
            s["dh"] = (torch.randn(M, K, device=DEV, generator=gen) * 0.02).bfloat16() if case["dh"] else None
            h = s.pop("x").float()
            s["rstd"] = torch.rsqrt(h.square().mean(1) + EPS)
            s["hq"], s["hs"] = _e4m3(h, case["ckpt"])
    return s


# ---- plain forms, in 32 bits

def _mx(x):
    """[rows, K] -> values of the 4-bit codes [rows, Kp / 32, 32] and their exponents [rows, Kp / 32, 1]."""
    g = torch.nn.functional.pad(x, (0, _padded(x.shape[1]) - x.shape[1])).view(x.shape[0], -1, GROUP)
    amax = g.abs().amax(-1, keepdim=True)
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 3, -127).clamp_min(-127)
    a = g * ((127 - e) << 23).view(torch.float32)
    m = a.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    return (torch.round(m / step) * step).clamp_max(6.0) * torch.where(a < 0, -1.0, 1.0), e


def _pack(v, e):
    """Codes two a byte (the first in the low half) and the exponents' bytes, as the framework stores them."""
    table = torch.tensor([0, 1, 2, 3, 4, 0, 5, 0, 6, 0, 0, 0, 7], dtype=torch.uint8, device=v.device)
    c = (table[(v.abs() * 2).to(torch.int64)] | ((v < 0).to(torch.uint8) << 3)).view(v.shape[0], -1, 2)
    return c[..., 0] | (c[..., 1] << 4), (e + 127).to(torch.uint8).view(v.shape[0], -1)


def _unpack(q, s):
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=q.device)
    v = table[torch.stack((q & 15, q >> 4), -1).to(torch.int32)].view(q.shape[0], -1, GROUP)
    return _scaled(v, s.to(torch.int32).unsqueeze(-1) - 127)


def _scaled(v, e):
    return (v / ((127 - e) << 23).view(torch.float32)).view(v.shape[0], -1)


def _mx_values(x):
    return _scaled(*_mx(x))


def _e4m3(x, mode):
    """Codes and scales: amax / 448 of each row, or of each 128 columns (power-of-two scales: the smallest that fits)."""
    g = x.view(x.shape[0], 1, -1) if mode == "row" else x.view(x.shape[0], -1, 128)
    amax = g.abs().amax(-1, keepdim=True).clamp_min(1e-12)
    if mode == "block_pow2":
        m, e = torch.frexp(amax)
        scale = torch.ldexp(torch.ones_like(amax), e - 9 + (m > 0.875).int())
        t = g / scale
    else:
        scale, t = amax / 448.0, g * (448.0 / amax)
    return t.clamp(-448.0, 448.0).view_as(x).to(torch.float8_e4m3fn), scale.view(-1) if mode == "row" else scale.view(x.shape[0], -1)


def _e4m3_values(q, s):
    return (q.float().view(q.shape[0], s.shape[1] if s.dim() == 2 else 1, -1) * s.view(q.shape[0], -1, 1)).view(q.shape)


def _run_plain(s):
    op = s["op"]
    if op == "requant":
        x = s["x"].float()
        v = _mx_values(x.t() if s["transpose"] else x)
        return v[:, :s["M"] if s["transpose"] else s["K"]].bfloat16()
    if op == "linear":
        x, w = _mx_values(s["x"].float()), _unpack(s["wq"], s["sw"])
        b = s["batch"]
        y = torch.bmm(x.view(b, s["M"], -1), w.view(b, s["N"], -1).transpose(1, 2).contiguous())
        return y.view(b * s["M"], s["N"]).bfloat16()
    if op == "train":
        x, w, dy = s["x"].float(), s["w"].float(), s["dy"].float()
        y = _mx_values(x) @ _mx_values(w.t()).t()
        dx = _mx_values(dy) @ _mx_values(w).t()
        dw = _mx_values(x.t()) @ _mx_values(dy.t()).t()
        return {"y": y.bfloat16(), "dx": dx.bfloat16(), "dw": dw}
    if op == "norm":
        h = s["x"].float() if s["res"] is None else s["x"].float() + s["res"].float()
        rstd = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
        y = h * rstd * s["gamma"].float()
        got = {"h": h.bfloat16() if s["res"] is not None else None, "rstd": rstd.view(-1) if s["ckpt"] else None}
        if s["out"] == "bf16":
            got["y"] = y.bfloat16()
        else:
            got["codes"], got["scales"] = _e4m3(y, s["out"])
        if s["ckpt"]:
            got["ckpt_codes"], got["ckpt_scales"] = _e4m3(h, "block")
        return got
    n = _e4m3_values(s["hq"], s["hs"]) * s["rstd"].view(-1, 1)
    dy = s["dy"].float()
    g = dy * s["gamma"].float()
    dx = s["rstd"].view(-1, 1) * (g - n * (g * n).mean(1, keepdim=True))
    return {"dx": (dx if s["dh"] is None else dx + s["dh"].float()).bfloat16(), "dgamma": (dy * n).sum(0)}


# ---- the framework's calls

def _run_own(s):
    from paper_2605_10886_amd import binding as B

    modes = {"row": B.SCALE_ROW, "block": B.SCALE_BLOCK_1x128, "block_pow2": B.SCALE_BLOCK_1x128_POW2}
    f8 = torch.float8_e4m3fn
    op, M, K = s["op"], s["M"], s["K"]
    if op == "requant":
        q, e = B.loka_mxfp4_quantize(s["x"], s["transpose"])
        return B.loka_mxfp4_dequantize(q, e, M if s["transpose"] else K)
    if op == "linear":
        d = B.make_mxfp4_desc(M, s["N"], K, s["batch"])
        if s["batch"] == 1:
            return B.loka_mxfp4_linear(d, s["x"], s["wq"], s["sw"])[0]
        xq, sx = B.loka_mxfp4_quantize(s["x"])
        return B.loka_mxfp4_gemm(d, xq, sx, s["wq"], s["sw"])[0]
    if op == "train":
        N, x, w, dy = s["N"], s["x"], s["w"], s["dy"]
        y, _ = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K), *B.loka_mxfp4_quantize(x), *B.loka_mxfp4_quantize(w, True))
        dx, _ = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, K, N), *B.loka_mxfp4_quantize(dy), *B.loka_mxfp4_quantize(w))
        _, dw = B.loka_mxfp4_gemm(B.make_mxfp4_desc(K, N, M), *B.loka_mxfp4_quantize(x, True), *B.loka_mxfp4_quantize(dy, True),
                                  want_out=False, want_y=True)
        return {"y": y, "dx": dx, "dw": dw}
    if op == "norm":
        bf16 = s["out"] == "bf16"
        r = B.loka_add_rmsnorm(s["x"], s["res"], s["gamma"], EPS, out=B.RMS_OUT_BF16 if bf16 else B.RMS_OUT_E4M3,
                               out_mode=modes.get(s["out"], B.SCALE_ROW), ckpt_mode=B.SCALE_BLOCK_1x128 if s["ckpt"] else None)
        got = {"h": r.h, "rstd": r.rstd}
        if bf16:
            got["y"] = r.y
        else:
            got["codes"], got["scales"] = r.y.view(f8), r.scales
        if s["ckpt"]:
            got["ckpt_codes"], got["ckpt_scales"] = r.hq.view(f8), r.hs
        return got
    dx, dgamma = B.loka_rmsnorm_backward(s["dy"], s["hq"].view(torch.uint8), s["hs"], s["rstd"], s["gamma"], s["dh"], ckpt_mode=modes[s["ckpt"]])
    return {"dx": dx, "dgamma": dgamma}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without

def work(case):
    M, K, op = case["M"], case["K"], case["op"]
    if op == "requant":                 # read, 4-bit codes and scales, values
        return {"bytes": M * K * (2 + 0.5 + 1 / 32 + 2), "flops": 4.0 * M * K}
    if op == "linear":
        N, b = case["N"], case["batch"]
        return {"bytes": b * (2.0 * M * K + N * K * (0.5 + 1 / 32) + 2.0 * M * N), "flops": 2.0 * b * M * N * K}
    if op == "train":
        N = case["N"]
        return {"bytes": 2.0 * (M * K + K * N + M * N) + 2.0 * (M * N + M * K) + 4.0 * K * N, "flops": 6.0 * M * N * K}
    if op == "norm":
        n = 2 + (4 if case["residual"] else 0) + (2 if case["out"] == "bf16" else 1) + (1 if case["ckpt"] else 0)
        return {"bytes": float(n) * M * K, "flops": 8.0 * M * K}
    return {"bytes": float(5 + (2 if case["dh"] else 0)) * M * K, "flops": 10.0 * M * K}


# ---- the definitions in 64 bits

def _pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_mx(x):
    rows, k = x.shape
    full = torch.zeros(rows, -(-k // GROUP) * GROUP, dtype=torch.float64, device=x.device)
    full[:, :k] = x.double()
    g = full.reshape(-1, GROUP)
    top = g.abs().max(dim=1).values
    # floor(log2) of a positive binary64 is its exponent field
    e = torch.where(top > 0, (top.view(torch.int64) >> 52) - 1023 - 2, -127).clamp(min=-127)
    unit = _pow2(e)[:, None]
    a = g.abs() / unit
    index = torch.zeros_like(a, dtype=torch.int64)
    for i in range(7):                  # halves between neighbours; a tie goes to the even code
        mid = (_E2M1[i] + _E2M1[i + 1]) / 2
        index += (a > mid) if i % 2 == 0 else (a >= mid)
    v = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)[index]
    return (torch.sign(g) * v * unit).reshape(rows, -1)[:, :k]


def _exact_weights(q, s, k):
    code = torch.empty(q.shape[0], q.shape[1] * 2, dtype=torch.int64, device=q.device)
    code[:, 0::2], code[:, 1::2] = (q % 16).long(), (q // 16).long()
    v = torch.tensor(_E2M1, dtype=torch.float64, device=q.device)[code % 8] * (1 - 2 * (code // 8)).double()
    return (v * _pow2(s.long() - 127).repeat_interleave(GROUP, dim=1))[:, :k]


def _exact_e4m3(x, mode):
    rows, k = x.shape
    width = k if mode == "row" else 128
    g = x.reshape(-1, width)
    top = g.abs().max(dim=1, keepdim=True).values.clamp(min=1e-12)
    scale = top / 448
    if mode == "block_pow2":
        m, e = torch.frexp(scale)       # the smallest power of two that is not less
        scale = _pow2(torch.where(m == 0.5, e - 1, e))
    t = g / scale
    # steps of 2^(exponent - 3), none below 2^-9
    step = _pow2((t.abs().clamp(min=2.0 ** -6).view(torch.int64) >> 52) - 1023 - 3)
    v = (torch.round(t / step) * step).clamp(-448, 448)
    return v.reshape(rows, k), scale.reshape(-1) if mode == "row" else scale.reshape(rows, -1)


def exact(case, seed):
    s = prepare(case, seed)
    op, M, K = case["op"], case["M"], case["K"]
    if op == "requant":
        return _exact_mx(s["x"].t().contiguous() if case["transpose"] else s["x"])
    if op == "linear":
        x, w = _exact_mx(s["x"]), _exact_weights(s["wq"], s["sw"], K)
        N = case["N"]
        return torch.cat([x[b * M:(b + 1) * M] @ w[b * N:(b + 1) * N].t() for b in range(case["batch"])])
    if op == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        turned = lambda t: _exact_mx(t.t().contiguous())
        return {"y": _exact_mx(x) @ turned(w).t(), "dx": _exact_mx(dy) @ _exact_mx(w).t(), "dw": turned(x) @ turned(dy).t()}
    gamma = s["gamma"].double()
    if op == "norm":
        h = s["x"].double() + (s["res"].double() if case["residual"] else 0)
        rstd = 1 / torch.sqrt((h * h).sum(1) / K + EPS)
        y = h * rstd[:, None] * gamma
        got = {"h": h if case["residual"] else None, "rstd": rstd if case["ckpt"] else None}
        if case["out"] == "bf16":
            got["y"] = y
        else:
            got["codes"], got["scales"] = _exact_e4m3(y, case["out"])
        if case["ckpt"]:
            got["ckpt_codes"], got["ckpt_scales"] = _exact_e4m3(h, "block")
        return got
    rstd, dy = s["rstd"].double()[:, None], s["dy"].double()
    hs = s["hs"].double().reshape(M, -1)
    h = s["hq"].double() * hs.repeat_interleave(K // hs.shape[1], dim=1)
    inner = (dy * gamma * h).sum(1, keepdim=True) * rstd / K
    dx = rstd * (dy * gamma - h * rstd * inner)
    return {"dx": dx if s["dh"] is None else dx + s["dh"].double(), "dgamma": (dy * h * rstd).sum(0)}
