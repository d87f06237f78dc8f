"""Plain 64-bit forms of a layer of experts, for the tests (test infrastructure, torch only; nothing here calls the library).

Roundings are counted in half steps: bf16 2^-8, fp32 2^-24, e4m3 2^-4 of the value."""
from __future__ import annotations

import math

import torch

import plain_ops as P

BLOCK = 128


# ---- the choice

def choose(logits, k):
    """Indices of the k greatest entries of each row (NaN above all, ties to the lower index), -1 where only minus infinities are left."""
    T, E = logits.shape
    x = logits.double()
    rank = torch.where(torch.isnan(x), math.inf, x)
    left = torch.ones(T, E, dtype=torch.bool, device=x.device) & (x != -math.inf)
    first_nan = torch.isnan(x)
    out = torch.full((T, k), -1, dtype=torch.int64, device=x.device)
    at = torch.arange(E, device=x.device).expand(T, E)
    for j in range(k):
        nan = left & first_nan
        pool = torch.where(nan.any(1, keepdim=True), nan, left)
        top = torch.where(pool, rank, -math.inf).amax(1, keepdim=True)
        best = torch.where(pool & (rank == top), at, E).amin(1)
        some = best < E
        out[:, j] = torch.where(some, best, -1)
        left[torch.arange(T, device=x.device)[some], best[some]] = False
    return out


def weights(logits, experts, score, renorm, scale=1.0):
    """The chosen experts' weights, differentiable in the logits."""
    x, live = logits.double(), experts >= 0
    mine = x.gather(1, experts.clamp_min(0))
    if score == "softmax":
        if renorm:
            w = torch.softmax(torch.where(live, mine, -math.inf), 1)
        else:
            w = torch.softmax(x, 1).gather(1, experts.clamp_min(0))
    elif renorm:
        # sigmoid ratios through their logarithms: none vanishes
        w = torch.softmax(torch.where(live, torch.nn.functional.logsigmoid(mine), -math.inf), 1)
    else:
        w = torch.sigmoid(mine)
    return torch.where(live, scale * w, 0.0)


def order(experts, E):
    """slots, rows and offsets of the routed order."""
    T, k = experts.shape
    slots, rows, offsets = torch.full((T, k), -1), [], [0]
    host = experts.cpu()
    for e in range(E):
        for t, j in (host == e).nonzero().tolist():
            slots[t, j] = len(rows)
            rows.append(t)
        offsets.append(len(rows))
    rows += [-1] * (T * k - len(rows))
    i32 = dict(dtype=torch.int32, device=experts.device)
    return slots.to(**i32), torch.tensor(rows, **i32), torch.tensor(offsets, **i32)


def order_of_many(experts, E):
    """The same by sorting, for many tokens."""
    T, k = experts.shape
    flat = torch.where(experts < 0, E, experts).reshape(-1)
    place = torch.sort(flat, stable=True).indices              # (tokens, and a token's choices, stay in their order)
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    n = int(counts.sum())
    slots, rows = torch.full_like(flat, -1), torch.full_like(flat, -1)
    slots[place[:n]] = torch.arange(n, device=flat.device)
    rows[:n] = place[:n] // k
    return slots.view(T, k).int(), rows.int(), torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()


# ---- stored forms

def _codes(v):
    """Values [..., 128] fp64 -> code values and scale [..., 1]; NaN scale and zero codes where one is not finite."""
    finite = torch.isfinite(v).all(-1, keepdim=True)
    v = torch.where(finite, v, 0.0)
    t = v.abs().amax(-1, keepdim=True).clamp_min(float(torch.tensor(1e-12))) / 448
    e = P.exponent(t)
    s = P.pow2(e)
    s = torch.where(s < t, 2 * s, s)
    a = v / s
    step = P.e4m3_step(a)
    return torch.round(a / step) * step, torch.where(finite, s, math.nan)


def along(x):
    """[rows, cols] -> code values [rows, colsp], scales [rows, colsp / 128]."""
    rows, cols = x.shape
    full = torch.zeros(rows, -(-cols // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    full[:, :cols] = x.double()
    c, s = _codes(full.view(rows, -1, BLOCK))
    return c.view(rows, -1), s.squeeze(-1)


def turned(x, offsets):
    """[rows, cols], group boundaries (a list) -> code values [blocks, cols, 128], scales [blocks, cols]; the blocks in use."""
    codes, scales = [], []
    for a, b in zip(offsets[:-1], offsets[1:]):
        for r in range(a, b, BLOCK):
            part = torch.zeros(x.shape[1], BLOCK, dtype=torch.float64, device=x.device)
            n = min(b, r + BLOCK) - r
            part[:, :n] = x[r:r + n].double().t()
            c, s = _codes(part)
            codes.append(c)
            scales.append(s.squeeze(-1))
    if not codes:
        return torch.zeros(0, x.shape[1], BLOCK, device=x.device).double(), torch.zeros(0, x.shape[1], device=x.device).double()
    return torch.stack(codes), torch.stack(scales)


def along_values(codes, scales, cols):
    v = codes.double().view(codes.shape[0], -1, BLOCK) * scales.double().unsqueeze(-1)
    return v.view(codes.shape[0], -1)[:, :cols]


def turned_values(codes, scales, count):
    """Codes [blocks, cols, 128] of ONE group of `count` rows -> [count, cols]."""
    v = codes.double() * scales.double().unsqueeze(-1)
    return v.permute(0, 2, 1).reshape(-1, codes.shape[1])[:count]


def e4m3(codes):
    return codes.view(torch.float8_e4m3fn).double()


# ---- bounds

def powers(v):
    """2^exponent of the value a code times its scale stands for (subnormal codes are far below what the tests hold): what the matrix
    instruction aligns a product's bits to."""
    a = v.abs()
    return torch.where(a > 0, P.pow2(P.exponent(torch.where(a > 0, a, 1.0))), 0.0)


def product_bound(xv, wv, terms):
    """Bound of |fp32 result - exact| of xv [M, K] @ wv [K, N]: the instruction keeps, of 8 products at a time, the bits down to 2^-13 of
    the largest power of two among them (8 of them lost at most: 2^-10 of that power, itself no more than the sum of the powers), and
    rounds each of the terms / 8 sums to fp32, as often again where partial sums join."""
    return 2.0 ** -10 * (powers(xv) @ powers(wv)) + (terms / 8 + 64) * P.F32 * (xv.abs() @ wv.abs())


# ---- sums

def combine(y, slots, w=None, residual=None):
    live = slots >= 0
    v = y.double()[slots.clamp_min(0).long()] * live.unsqueeze(-1)
    if w is not None:
        v = v * w.double().unsqueeze(-1)
    out = v.sum(1)
    return out if residual is None else out + residual.double()


def combine_backward(dout, y, slots, w, rows):
    live = slots >= 0
    d = dout.double()
    dy = torch.zeros(rows, d.shape[1], dtype=torch.float64, device=d.device)
    for j in range(slots.shape[1]):
        on = live[:, j]
        dy[slots[on, j].long()] = d[on] * (1.0 if w is None else w[on, j:j + 1].double())
    dw = (d.unsqueeze(1) * y.double()[slots.clamp_min(0).long()]).sum(-1) * live
    return dy, dw
