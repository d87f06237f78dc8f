"""The operators of a layer of experts, as cases that can be timed and compared.

A layer of experts sends each token to `top_k` of `experts` linear layers, which hold 8-bit weights with a power-of-two
scale per 128 elements.  The (token, choice) pairs lie sorted by expert ("routed order"); expert e owns rows
offsets[e] .. offsets[e + 1] - 1, as many as chose it.  A case is one pass through the Python binding:

  route     loka_route: the choice, its weights, and the routed order; a training step also takes loka_route_backward
  quantize  loka_grouped_quantize: a matrix to 8-bit codes in both stored forms (along its rows, and turned: down its
            columns, 128 rows of one group to a scale), of weights or of rows gathered into the routed order
  linear    loka_grouped_linear: bf16 tokens through the experts' kept weights
  train     one training step of the experts: forward, dX = dY W^T, dW = X^T dY, every operand quantized in the step
  combine   loka_combine: the weighted sum of a token's results, and loka_combine_backward in training

Activations are N(0, 1), Student-t(4) / sqrt 2 (heavy tails) or N(0, 1) with four channels x 100 (outliers), weights
N(0, 1/K), output gradients N(0, 0.02^2), router logits N(0, 1.5^2) plus N(0, 0.7^2) for each expert (uneven loads); all
drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False
BLOCK = 128                             # elements that share a scale; what a stored row's length is a multiple of
DEV = "cuda"
F8 = torch.float8_e4m3fn


def _route(T, E, k, score="softmax", renorm=True, bf16=False, masked=False, train=False, **name):
    return dict(name, op="route", T=T, E=E, k=k, score=score, renorm=renorm, bf16=bf16, masked=masked, train=train)


def _quantize(T, E, k, K, gather=True, dist="normal", **name):
    return dict(name, op="quantize", T=T, E=E, k=k, K=K, gather=gather, dist=dist)


def _linear(T, E, k, K, N, dist="normal", **name):
    return dict(name, op="linear", T=T, E=E, k=k, K=K, N=N, dist=dist)


def _train(T, E, k, K, N, dist="normal", **name):
    return dict(name, op="train", T=T, E=E, k=k, K=K, N=N, dist=dist)


def _combine(T, E, k, K, residual=True, train=False, **name):
    return dict(name, op="combine", T=T, E=E, k=k, K=K, residual=residual, train=train)


def listed():
    return [
        # one token's choice while serving: latency
        _route(1, 64, 8, name="route_1x64"),
        # a training batch's choice and its gradient, in a router that scores by sigmoids
        _route(32768, 256, 8, score="sigmoid", bf16=True, train=True, name="route_32768x256_train"),
        # the experts' weights after an optimizer step: both forms, of 16 matrices of a mid-sized layer
        _quantize(16 * 1024, 16, 1, 4096, gather=False, name="quantize_16x1024x4096"),
        # a batch's activations gathered for the weight gradient: ragged groups and widths, heavy tails
        _quantize(5013, 23, 2, 1008, dist="student_t4", name="quantize_5013x1008"),
        # one token through eight of 64 experts: latency and weight traffic
        _linear(1, 64, 8, 1024, 4096, name="linear_1x1024x4096"),
        # a small batch of tokens through few widening experts: weight traffic
        _linear(13, 8, 2, 4096, 16384, dist="normal_outlier4", name="linear_13x4096x16384"),
        # feature widths, row counts and numbers of experts as they come
        _linear(5013, 23, 2, 1008, 720, dist="student_t4", name="linear_5013x1008x720"),
        # a large batch: as many products as the benchmark's headline layer, over 16 experts
        _linear(16384, 16, 2, 4096, 4096, dist="normal_outlier4", name="linear_16384x4096x4096"),
        # training steps: the narrowest layer of the throughput study at its batch of 2048, and a mid-sized layer
        _train(2048, 8, 2, 256, 768, name="train_2048x256x768"),
        _train(16384, 16, 2, 1024, 4096, dist="student_t4", name="train_16384x1024x4096"),
        # one token's sum while serving: latency
        _combine(1, 64, 8, 4096, name="combine_1x4096"),
        # a training batch's sum and its gradients
        _combine(16384, 64, 4, 4096, train=True, name="combine_16384x4096_train"),
    ]


def _log(rng, lo, hi):
    hi = max(lo, hi)
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dist = rng.choice(("normal", "student_t4", "normal_outlier4"))
    op = rng.choice(("route", "quantize", "linear", "linear", "train", "combine"))
    E = _log(rng, 1, 64)
    k = rng.randint(1, min(8, E))
    if op == "route":
        E = _log(rng, 4, 512)
        k = rng.randint(1, min(8, E))
        return _route(_log(rng, 1, 32768 * 256 // max(E, 64)), E, k, score=rng.choice(("softmax", "sigmoid")),
                      renorm=k > 1 and rng.random() < 0.6, bf16=rng.random() < 0.5, masked=rng.random() < 0.3, train=rng.random() < 0.5)
    if op == "quantize":
        if rng.random() < 0.3:          # weights
            K, rows = _log(rng, 64, 4096), _log(rng, 64, 1024)
            E = _log(rng, 1, min(64, (1 << 26) // (K * rows)))
            return _quantize(E * rows, E, 1, K, gather=False)
        K = _log(rng, 16, 4096)
        return _quantize(_log(rng, 1, min(16384, (1 << 26) // (K * k))), E, k, K, dist=dist)
    K, N = _log(rng, 64, 4096), _log(rng, 64, 4096)
    if op == "combine":
        return _combine(_log(rng, 1, min(16384, (1 << 28) // (K * k))), E, k, K, residual=rng.random() < 0.6, train=rng.random() < 0.5)
    while E * K * N > 1 << 28:
        K, N = max(64, K // 2), max(64, N - N // 3)
    if op == "linear":
        few = rng.random() < 0.5        # tokens of a serving batch
        return _linear(_log(rng, 1, 64) if few else _log(rng, 65, min(16384, (1 << 39) // (k * K * N))), E, k, K, N, dist=dist)
    return _train(_log(rng, 64, min(16384, (1 << 37) // (k * K * N))), E, k, K, N, dist=dist)


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


def _logits(T, E, gen):
    return 1.5 * torch.randn(T, E, device=DEV, generator=gen) + 0.7 * torch.randn(E, device=DEV, generator=gen)


def _blocks(rows, groups):
    """Blocks of 128 rows that `rows` rows in `groups` groups can take, each group beginning a block."""
    return (rows + 127 * min(rows, groups)) // BLOCK


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, E, k, op = case["T"], case["E"], case["k"], case["op"]
    s = dict(case)
    logits = _logits(T, E, gen)
    if op == "route":
        if case["masked"]:              # experts that a token may not take
            logits.masked_fill_(torch.rand(T, E, device=DEV, generator=gen) < 0.4, -math.inf)
        s["logits"] = logits.bfloat16() if case["bf16"] else logits
        s["dweights"] = torch.randn(T, k, device=DEV, generator=gen) if case["train"] else None
        return s
    K = case["K"]
    if op == "quantize" and not case["gather"]:
        s["x"] = (torch.randn(T, K, device=DEV, generator=gen) / math.sqrt(K)).bfloat16()
        s["offsets"] = s["index"] = None
        s["host"] = [e * (T // E) for e in range(E + 1)]
    else:
        r = _plain_route(logits, k, "softmax", True)
        s["weights"], s["slots"], s["index"], s["offsets"] = r["weights"], r["slots"], r["rows"], r["offsets"]
        s["host"] = s["offsets"].tolist()       # (read by the plain form alone)
    if op == "quantize":
        if case["gather"]:
            s["x"] = _values(T, K, case["dist"], gen)
        blocks = _blocks(T * k, E)
        s["qt"] = torch.zeros(blocks, K, BLOCK, dtype=torch.uint8, device=DEV)
        s["st"] = torch.zeros(blocks, K, device=DEV)
    elif op == "linear":
        s["x"] = _values(T, K, case["dist"], gen)
        codes, scales = [], []
        for _ in range(E):              # weights [K, N], kept turned: codes [K / 128, N, 128] and scales [K / 128, N]
            c, f = _turned((torch.randn(K, case["N"], device=DEV, generator=gen) / math.sqrt(K)).bfloat16().float())
            codes.append(c.view(torch.uint8))
            scales.append(f)
        s["wq"], s["sw"] = torch.cat(codes), torch.cat(scales)
    elif op == "train":
        s["x"] = _values(T, K, case["dist"], gen)
        s["w"] = (torch.randn(E * K, case["N"], device=DEV, generator=gen) / math.sqrt(K)).bfloat16()
        s["dy"] = (torch.randn(T * k, case["N"], device=DEV, generator=gen) * 0.02).bfloat16()
    else:
        s["y"] = torch.randn(T * k, K, device=DEV, generator=gen).bfloat16()
        s["res"] = torch.randn(T, K, device=DEV, generator=gen).bfloat16() if case["residual"] else None
        s["dout"] = (torch.randn(T, K, device=DEV, generator=gen) * 0.02).bfloat16() if case["train"] else None
    return s


# ---- plain forms, in 32 bits

def _plain_route(logits, k, score, renorm):
    T, E = logits.shape
    x = logits.float()
    value, order = torch.sort(x, dim=1, descending=True, stable=True)      # (ties: the lowest index first)
    value, chosen = value[:, :k], order[:, :k]
    live = value != -math.inf
    if score == "softmax":
        p = torch.exp(x - x.amax(1, keepdim=True).clamp_min(-3e38))
        w = torch.where(live, p.gather(1, chosen), 0.0)
        w = w / (w.sum(1, keepdim=True) if renorm else p.sum(1, keepdim=True)).clamp_min(1e-38)
    else:
        w = torch.where(live, torch.sigmoid(value), 0.0)
        if renorm:
            w = w / w.sum(1, keepdim=True).clamp_min(1e-38)
    experts = torch.where(live, chosen, -1)
    flat = torch.where(live, chosen, E).reshape(-1)
    place = torch.sort(flat, stable=True).indices                          # routed order -> token * k + choice
    slots = torch.empty_like(place)
    slots[place] = torch.arange(T * k, device=x.device)
    counts = (flat[:, None] == torch.arange(E, device=x.device)).sum(0) if T * k * E < 1 << 24 else torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=x.device)
    offsets[1:] = counts.cumsum(0)
    rows = torch.where(flat[place] < E, place // k, -1)
    i32 = torch.int32
    return {"experts": experts.to(i32), "weights": w, "slots": torch.where(live, slots.view(T, k), -1).to(i32), "rows": rows.to(i32), "offsets": offsets.to(i32)}


def _plain_route_backward(logits, r, g, score, renorm):
    x = logits.float()
    chosen, live = r["experts"].clamp_min(0).long(), r["experts"] >= 0
    g = torch.where(live, g, 0.0)
    d = torch.zeros_like(x)
    if score == "softmax":
        if renorm:
            t = r["weights"] * (g - (g * r["weights"]).sum(1, keepdim=True))
        else:
            p = torch.exp(x - x.amax(1, keepdim=True).clamp_min(-3e38))
            p = p / p.sum(1, keepdim=True).clamp_min(1e-38)
            inner = (g * r["weights"]).sum(1, keepdim=True)
            d = -p * inner
            t = g * r["weights"]
    else:
        sig = torch.sigmoid(x.gather(1, chosen))
        t = (r["weights"] * (g - (g * r["weights"]).sum(1, keepdim=True)) if renorm else g * sig) * (1 - sig)
    d.scatter_add_(1, chosen, torch.where(live, t, 0.0))
    return d.to(logits.dtype)


def _codes(g):
    """Codes of fp32 values [..., 128] and the power of two that their last axis shares: the least s with amax / s <= 448."""
    m, e = torch.frexp(g.abs().amax(-1, keepdim=True).clamp_min(1e-12))
    scale = ((e - 9 + (m > 0.875).int() + 127) << 23).view(torch.float32)
    return (g / scale).clamp(-448.0, 448.0).to(F8), scale


def _along(x):
    """x [rows, K] -> codes [rows, Kp] and scales [rows, Kp / 128]."""
    k = x.shape[1]
    q, s = _codes(torch.nn.functional.pad(x, (0, -k % BLOCK)).view(x.shape[0], -1, BLOCK))
    return q.view(x.shape[0], -1), s.view(x.shape[0], -1)


def _turned(x):
    """x [K, N] -> codes [Kp / 128, N, 128] and scales [Kp / 128, N]."""
    x = torch.nn.functional.pad(x, (0, 0, 0, -x.shape[0] % BLOCK))
    q, s = _codes(x.view(-1, BLOCK, x.shape[1]).transpose(1, 2).contiguous())
    return q, s.squeeze(-1)


def _along_values(x):
    q, s = _along(x)
    return (q.float().view(x.shape[0], -1, BLOCK) * s.unsqueeze(-1)).view(x.shape[0], -1)[:, :x.shape[1]]


def _turned_values(x):
    q, s = _turned(x)
    return _untangle(q, s)[:x.shape[0]]


def _untangle(q, s):
    """The values of turned codes, [Kp, N]."""
    return (q.float() * s.unsqueeze(-1)).transpose(1, 2).reshape(-1, s.shape[1])


def _run_plain(s):
    op, E, host = s["op"], s["E"], s.get("host")
    if op == "route":
        r = _plain_route(s["logits"], s["k"], s["score"], s["renorm"])
        if s["train"]:
            r["dlogits"] = _plain_route_backward(s["logits"], r, s["dweights"], s["score"], s["renorm"])
        return r
    if op == "combine":
        slots = s["slots"].long()
        y = s["y"].float()[slots]
        out = (y * s["weights"].unsqueeze(-1)).sum(1)
        got = {"out": (out if s["res"] is None else out + s["res"].float()).bfloat16()}
        if s["train"]:
            dout = s["dout"].float().unsqueeze(1)
            got["dweights"] = (dout * y).sum(-1)
            dy = torch.empty(s["y"].shape, device=DEV)
            dy[slots.view(-1)] = (dout * s["weights"].unsqueeze(-1)).view(-1, s["K"])
            got["dy"] = dy.bfloat16()
        return got
    spans = [(e, host[e], host[e + 1]) for e in range(E) if host[e + 1] > host[e]]
    if op == "quantize":
        x = s["x"].float()
        if s["gather"]:
            x = x[s["index"].long()]
        q, f = _along(x)
        at = 0
        for _, a, b in spans:
            c, t = _turned(x[a:b])
            s["qt"][at:at + len(c)], s["st"][at:at + len(c)] = c.view(torch.uint8), t
            at += len(c)
        return {"codes": q, "scales": f, "turned_codes": s["qt"].view(F8), "turned_scales": s["st"]}
    N, K = s["N"], s["K"]
    x, index = s["x"].float(), s["index"].long()
    y = torch.empty(len(index), N, dtype=torch.bfloat16, device=DEV)
    xv = _along_values(x)
    if op == "linear":
        nb = -(-K // BLOCK)
        for e, a, b in spans:
            w = _untangle(s["wq"][e * nb:(e + 1) * nb].view(F8), s["sw"][e * nb:(e + 1) * nb])[:K]
            y[a:b] = (xv[index[a:b]] @ w).bfloat16()
        return y
    dx = torch.empty(len(index), K, dtype=torch.bfloat16, device=DEV)
    dw = torch.zeros(E, K, N, dtype=torch.bfloat16, device=DEV)
    dy = s["dy"].float()
    dyv = _along_values(dy)
    for e, a, b in spans:
        w = s["w"][e * K:(e + 1) * K].float()
        y[a:b] = (xv[index[a:b]] @ _turned_values(w)).bfloat16()
        dx[a:b] = (dyv[a:b] @ _along_values(w).t().contiguous()).bfloat16()
        dw[e] = (_turned_values(x[index[a:b]]).t().contiguous() @ _turned_values(dy[a:b])).bfloat16()
    return {"y": y, "dx": dx, "dw": dw}


# ---- the framework's calls

def _run_own(s):
    from paper_2605_10886_amd import binding as B

    op, E = s["op"], s["E"]
    if op == "route":
        score = B.SCORE_SOFTMAX if s["score"] == "softmax" else B.SCORE_SIGMOID
        r = B.loka_route(s["logits"], s["k"], score=score, renorm=s["renorm"])
        got = r._asdict()
        if s["train"]:
            got["dlogits"] = B.loka_route_backward(s["logits"], r.experts, s["dweights"], score=score, renorm=s["renorm"])
        return got
    if op == "combine":
        got = {"out": B.loka_combine(s["y"], s["slots"], s["weights"], residual=s["res"])}
        if s["train"]:
            got["dy"], got["dweights"] = B.loka_combine_backward(s["dout"], s["y"], s["slots"], s["weights"])
        return got
    if op == "quantize":
        r = B.loka_grouped_quantize(s["x"], groups=E, offsets=s["offsets"], index=s["index"], turned=True, qt=s["qt"], st=s["st"])
        return {"codes": r.q.view(F8), "scales": r.scales, "turned_codes": r.qt.view(F8), "turned_scales": r.st}
    T, k, K, N, offsets, index = s["T"], s["k"], s["K"], s["N"], s["offsets"], s["index"]
    forward = B.make_grouped_desc(T * k, N, K, E)
    if op == "linear":
        return B.loka_grouped_linear(forward, s["x"], s["wq"], s["sw"], offsets, index=index)[0]
    w = B.loka_grouped_quantize(s["w"], groups=E, turned=True)
    x = B.loka_grouped_quantize(s["x"])
    xt = B.loka_grouped_quantize(s["x"], offsets=offsets, index=index, along=False, turned=True)
    dy = B.loka_grouped_quantize(s["dy"], offsets=offsets, turned=True)
    y, _ = B.loka_grouped_gemm(forward, x.q, x.scales, w.qt, w.st, offsets, index=index)
    dx, _ = B.loka_grouped_gemm(B.make_grouped_desc(T * k, K, N, E, turned_w=False), dy.q, dy.scales, w.q, w.scales, offsets)
    dw, _ = B.loka_grouped_wgrad(forward, xt.qt, xt.st, dy.qt, dy.st, offsets)
    return {"y": y, "dx": dx, "dw": dw}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without

def work(case):
    T, E, k, op = case["T"], case["E"], case["k"], case["op"]
    R = T * k
    if op == "route":
        size = 2 if case["bf16"] else 4
        n = T * E * size + R * 16 + 4 * (E + 1)
        return {"bytes": float(n + (T * E * 2 * size + R * 8 if case["train"] else 0)), "flops": float(T * E * (12 if case["train"] else 6))}
    K = case["K"]
    if op == "quantize":                # read, and two times codes and scales
        return {"bytes": 2.0 * T * K + 2.0 * (1 + 1 / 32) * R * K, "flops": 6.0 * R * K}
    if op == "combine":
        n = R * K * 2 + T * K * (4 if case["residual"] else 2) + R * 8
        return {"bytes": float(n + (R * K * 4 + T * K * 2 + R * 12 if case["train"] else 0)), "flops": float(R * K * (5 if case["train"] else 2))}
    N = case["N"]
    used = E * (1 - (1 - k / E) ** T)   # experts that a token takes, were the loads even
    if op == "linear":
        return {"bytes": 2.0 * T * K + used * N * K * (1 + 1 / 32) + 2.0 * R * N, "flops": 2.0 * R * N * K}
    return {"bytes": 2.0 * (T * K + E * K * N + R * N) + 2.0 * (R * N + R * K + E * K * N), "flops": 6.0 * R * N * K}


# ---- the definitions in 64 bits

def _pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_groups(v):
    """Values that the codes of v [n, <= 128] (fp64) stand for, code values and scale."""
    top = v.abs().max(dim=1, keepdim=True).values.clamp(min=1e-12)
    bits = (top / 448).view(torch.int64)
    up = (bits & ((1 << 52) - 1)) != 0   # the least power of two that is not less
    scale = _pow2((bits >> 52) - 1023 + up)
    t = v / scale
    step = _pow2((t.abs().clamp(min=2.0 ** -6).view(torch.int64) >> 52) - 1023 - 3)
    return (torch.round(t / step) * step).clamp(-448, 448), scale


def _exact_rows(x):
    """[rows, K] fp64 -> code values [rows, Kp], scales [rows, Kp / 128]."""
    rows, k = x.shape
    full = torch.zeros(rows, -(-k // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    full[:, :k] = x
    c, s = _exact_groups(full.reshape(-1, BLOCK))
    return c.reshape(rows, -1), s.reshape(rows, -1)


def _exact_value(x):
    c, s = _exact_rows(x)
    return (c * s.repeat_interleave(BLOCK, dim=1))[:, :x.shape[1]]


def _exact_route(case, s):
    x = s["logits"].double()
    T, E = x.shape
    k = case["k"]
    left, chosen, live = x.clone(), [], []
    low = torch.arange(E, device=x.device).expand(T, E)
    for _ in range(k):
        top = left.max(dim=1, keepdim=True).values
        i = torch.where(left == top, low, E).min(dim=1, keepdim=True).values
        chosen.append(i)
        live.append(top > -math.inf)
        left.scatter_(1, i, -math.inf)
    chosen, live = torch.cat(chosen, 1), torch.cat(live, 1)
    if case["score"] == "softmax":
        share = torch.nan_to_num(torch.softmax(x, 1))
    else:
        share = 1 / (1 + torch.exp(-x))
    own_share = share.gather(1, chosen) * live
    total = own_share.sum(1, keepdim=True)
    w = own_share / torch.where(total > 0, total, 1.0) if case["renorm"] else own_share
    taken = torch.zeros(T, E, dtype=torch.int64, device=x.device)
    taken.scatter_add_(1, chosen, live.long())
    counts = taken.sum(0)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    before = taken.cumsum(0) - taken     # earlier tokens of the same expert
    slots = torch.where(live, offsets[:-1][chosen] + before.gather(1, chosen), -1)
    rows = torch.full((T * k,), -1, dtype=torch.int64, device=x.device)
    rows[slots[live]] = torch.arange(T, device=x.device)[:, None].expand(T, k)[live]
    i32 = torch.int32
    got = {"experts": torch.where(live, chosen, -1).to(i32), "weights": w, "slots": slots.to(i32), "rows": rows.to(i32), "offsets": offsets.to(i32)}
    if case["train"]:
        g = s["dweights"].double() * live
        dshare = torch.zeros_like(x)
        if case["renorm"]:
            g = (g - (g * w).sum(1, keepdim=True)) / torch.where(total > 0, total, 1.0)
        dshare.scatter_add_(1, chosen, g * live)
        if case["score"] == "softmax":
            got["dlogits"] = share * (dshare - (dshare * share).sum(1, keepdim=True))
        else:
            got["dlogits"] = dshare * share * (1 - share)
    return got


def exact(case, seed):
    s = prepare(case, seed)
    op, E = case["op"], case["E"]
    if op == "route":
        return _exact_route(case, s)
    if op == "combine":
        T, k, K = case["T"], case["k"], case["K"]
        out = torch.zeros(T, K, dtype=torch.float64, device=DEV) if s["res"] is None else s["res"].double()
        dw = torch.empty(T, k, dtype=torch.float64, device=DEV)
        dy = torch.empty(T * k, K, dtype=torch.float64, device=DEV) if case["train"] else None
        for j in range(k):
            at, w = s["slots"][:, j].long(), s["weights"][:, j:j + 1].double()
            mine = s["y"][at].double()
            out = out + w * mine
            if case["train"]:
                dw[:, j] = (s["dout"].double() * mine).sum(1)
                dy[at] = w * s["dout"].double()
        return {"out": out, "dy": dy, "dweights": dw} if case["train"] else {"out": out}
    bound = s["host"]
    index = s["index"].long() if s["index"] is not None else torch.arange(case["T"], device=DEV)
    if op == "quantize":
        x = s["x"].double()[index]
        c, f = _exact_rows(x)
        qt, st = torch.zeros(s["qt"].shape, dtype=torch.float64, device=DEV), torch.zeros(s["st"].shape, dtype=torch.float64, device=DEV)
        b = 0
        for e in range(E):
            for a in range(bound[e], bound[e + 1], BLOCK):
                part = x[a:min(a + BLOCK, bound[e + 1])].t().contiguous()
                v, sc = _exact_groups(part)
                qt[b, :, :part.shape[1]], st[b] = v, sc[:, 0]
                b += 1
        return {"codes": c, "scales": f, "turned_codes": qt, "turned_scales": st}
    K, N = case["K"], case["N"]
    xv = _exact_value(s["x"].double())
    y = torch.zeros(len(index), N, dtype=torch.float64, device=DEV)
    if op == "linear":
        nb = s["wq"].shape[0] // E
        for e in range(E):
            if bound[e + 1] > bound[e]:
                w = s["wq"][e * nb:(e + 1) * nb].view(F8).double() * s["sw"][e * nb:(e + 1) * nb].double()[:, :, None]
                w = w.permute(0, 2, 1).reshape(-1, N)[:K]
                y[bound[e]:bound[e + 1]] = xv[index[bound[e]:bound[e + 1]]] @ w
        return y
    dx = torch.zeros(len(index), K, dtype=torch.float64, device=DEV)
    dw = torch.zeros(E, K, N, dtype=torch.float64, device=DEV)
    down = lambda m: torch.cat([_exact_value(p.t().contiguous()).t() for p in m.split(BLOCK)])     # scales down the columns
    dyv = _exact_value(s["dy"].double())
    for e in range(E):
        a, b = bound[e], bound[e + 1]
        if b > a:
            w = s["w"][e * K:(e + 1) * K].double()
            y[a:b] = xv[index[a:b]] @ down(w)
            dx[a:b] = dyv[a:b] @ _exact_value(w).t()
            dw[e] = down(s["x"].double()[index[a:b]]).t() @ down(s["dy"][a:b].double())
    return {"y": y, "dx": dx, "dw": dw}
