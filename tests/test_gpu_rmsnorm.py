"""Residual addition + RMSNorm + quantization and its backward pass from the 8-bit checkpoint, against plain 64-bit forms."""
import pytest
import torch

import plain_ops as P
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MODES = {"row": B.SCALE_ROW, "block": B.SCALE_BLOCK_1x128, "pow2": B.SCALE_BLOCK_1x128_POW2}


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _inputs(rows, cols, seed, residual=True, gamma=True):
    g = _gen(seed)
    x = torch.randn(rows, cols, device=DEV, generator=g)
    x[:, ::97] *= 50.0
    r = torch.randn(rows, cols, device=DEV, generator=g).bfloat16() if residual else None
    w = (1 + 0.2 * torch.randn(cols, device=DEV, generator=g)).bfloat16() if gamma else None
    return x.bfloat16(), r, w


# fp32 roundings between the inputs and y, relative: the sum of squares adds at most 64 terms in a thread, 6 exchanges and 16
# waves, and each square and h itself are rounded (rstd has half of that), then division, root, mean and the products with
# rstd, gamma and the scale's factors
REL = ((64 + 6 + 16 + 3) / 2 + 10) * P.F32


def _check_e4m3(q, s, v, mode, what):
    """Codes and scales of the fp64 matrix v: scales within REL of amax / 448 (power-of-two modes: one of the two neighbours where
    amax is within REL of the border), each code a value nearest to v / scale, up to REL."""
    rows, cols = v.shape
    g = v.reshape(rows, 1, cols) if mode == "row" else v.reshape(rows, -1, 128)
    amax = g.abs().amax(-1).clamp_min(1e-12)
    got = s.double().view_as(amax)
    if mode == "pow2":
        assert torch.equal(got, P.pow2(P.exponent(got))), what
        fits = amax / got
        assert bool((fits <= 448 * (1 + REL)).all()) and bool((fits * 2 > 448 * (1 - REL)).all()), what
    else:
        assert bool(((got - amax / 448).abs() <= REL * amax / 448).all()), what
    t = (g / got[..., None]).reshape(rows, cols)
    err = (P.e4m3_values(q).view(rows, cols) - t.clamp(-448, 448)).abs()
    tol = P.e4m3_step(t) / 2 + 2 * REL * t.abs()
    assert bool((err <= tol).all()), (what, float((err / tol).max()))


SHAPES = [(1, 16), (1, 4096), (3, 128), (5, 208), (64, 256), (33, 512), (17, 640), (9, 1008), (130, 1024), (4, 2048), (300, 4096), (7, 4112), (3, 8192),
          (2, 16384), (5, 16400), (2, 32768), (1000, 128), (2050, 128), (2049, 240), (2060, 512), (2048, 1008), (2051, 1920), (2053, 4096)]


@pytest.mark.parametrize("residual,gamma", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_bf16_output(rows, cols, residual, gamma):
    x, r, w = _inputs(rows, cols, rows + cols, residual, gamma)
    got = B.loka_add_rmsnorm(x, r, w, 1e-5, out=B.RMS_OUT_BF16, want_rstd=True)
    h, rstd, y = P.rms_forward(x, r, w, 1e-5)
    assert got.scales is None and got.hq is None and got.hs is None
    assert bool(((got.rstd.double() - rstd.view(-1)).abs() <= REL * rstd.view(-1)).all())
    assert bool(((got.y.double() - y).abs() <= (2.0 ** -8 + REL) * y.abs()).all())
    if residual:
        assert torch.equal(got.h, (x.float() + r.float()).bfloat16())
    else:
        assert got.h is None


@pytest.mark.parametrize("rows,cols,mode,ckpt",
                         [(*s, m, c) for s in SHAPES if s[1] % 128 == 0 for m in MODES for c in (None, *MODES)] +
                         [(*s, "row", c) for s in ((5, 208), (9, 1008), (3, 16400)) for c in (None, "row")])
def test_e4m3_output_and_checkpoint(rows, cols, mode, ckpt):
    x, r, w = _inputs(rows, cols, rows + 3 * cols, residual=rows % 2 == 1)
    got = B.loka_add_rmsnorm(x, r, w, 1e-5, out_mode=MODES[mode], ckpt_mode=None if ckpt is None else MODES[ckpt])
    h, _, y = P.rms_forward(x, r, w, 1e-5)
    _check_e4m3(got.y, got.scales, y, mode, "y")
    if ckpt is None:
        assert got.hq is None and got.hs is None and got.rstd is None
        return
    _check_e4m3(got.hq, got.hs, h, ckpt, "checkpoint")
    if r is None:                      # the recipe is loka_quantize's, to the bit
        q, s = B.loka_quantize(x, MODES[ckpt])
        assert torch.equal(got.hq, q) and torch.equal(got.hs.view(-1), s)


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_mxfp4_output(rows, cols):
    x, r, w = _inputs(rows, cols, rows + 5 * cols)
    got = B.loka_add_rmsnorm(x, r, w, 1e-5, out=B.RMS_OUT_MXFP4)
    _, _, y = P.rms_forward(x, r, w, 1e-5)
    kp = P.padded(cols)
    assert got.y.shape == (rows, kp // 2) and got.scales.shape == (rows, kp // 32)
    g = torch.zeros(rows, kp, dtype=torch.float64, device=DEV)
    g[:, :cols] = y
    g = g.view(rows, -1, 32)
    amax = g.abs().amax(-1)
    byte = got.scales.long()
    lo, hi = (torch.where(amax > 0, P.exponent((amax * f).clamp_min(1e-300)) - 2, -127).clamp_min(-127) + 127 for f in (1 - REL, 1 + REL))
    assert bool(((byte >= lo) & (byte <= hi)).all())
    t = g / P.pow2(byte - 127)[..., None]
    v = P.mx_values(got.y, got.scales).view_as(g) / P.pow2(byte - 127)[..., None]
    step = torch.where(t.abs() < 2, 0.5, torch.where(t.abs() < 4, 1.0, 2.0))
    assert bool(((v - t.clamp(-6, 6)).abs() <= step / 2 + 2 * REL * t.abs()).all())
    assert not bool(v.reshape(rows, kp)[:, cols:].any())


def test_strides_and_in_place():
    rows, cols = 70, 384
    big, bigr = (torch.randn(rows, 400 + 8 * i, device=DEV, generator=_gen(i)).bfloat16() for i in (1, 2))
    x, r = big[:, 8:8 + cols], bigr[:, 16:16 + cols]
    w = torch.randn(cols, device=DEV, generator=_gen(3)).bfloat16()
    kw = dict(out_mode=B.SCALE_ROW, ckpt_mode=B.SCALE_BLOCK_1x128)
    a = B.loka_add_rmsnorm(x, r, w, **kw)
    b = B.loka_add_rmsnorm(x.contiguous(), r.contiguous(), w, **kw)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    for into in (0, 1):                # the sum over x or over the residual
        t = [x.contiguous(), r.contiguous()]
        c = B.loka_add_rmsnorm(*t, w, h_out=t[into], **kw)
        assert c.h.data_ptr() == t[into].data_ptr() and all(torch.equal(p, q) for p, q in zip(c, b))
    # the backward pass: strided gradients, dx over dy or dh
    dy, dh = big[:, 16:16 + cols], bigr[:, 8:8 + cols]
    ref = B.loka_rmsnorm_backward(dy.contiguous(), b.hq, b.hs, b.rstd, w, dh.contiguous())
    got = B.loka_rmsnorm_backward(dy, b.hq, b.hs, b.rstd, w, dh)
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])
    for into in (0, 1):
        t = [dy.contiguous(), dh.contiguous()]
        got = B.loka_rmsnorm_backward(t[0], b.hq, b.hs, b.rstd, w, t[1], dx=t[into])
        assert torch.equal(ref[0], t[into]) and torch.equal(ref[1], got[1])


def test_degenerate_rows():
    cols = 256
    x = torch.randn(8, cols, device=DEV, generator=_gen(1)).bfloat16()
    x[1] = 0
    x[2] = 1e-20                       # y far below the scales' floor
    x[3, 7], x[4, 9], x[5, 200] = float("nan"), float("inf"), float("-inf")
    x[6] = 1e15
    h, rstd, y = P.rms_forward(x, None, None, 1e-5)
    bad = torch.isnan(x).any(1) | torch.isinf(x).any(1)
    got = B.loka_add_rmsnorm(x, None, None, 1e-5, out=B.RMS_OUT_BF16)
    assert torch.equal(torch.isnan(got.y), torch.isnan(y)) and bool(((got.y.double() - y).abs()[~bad] <= (2.0 ** -8 + REL) * y.abs()[~bad]).all())
    for mode in MODES:
        got = B.loka_add_rmsnorm(x, None, None, 1e-5, out_mode=MODES[mode], ckpt_mode=MODES[mode])
        _check_e4m3(got.y[~bad], got.scales.view(8, -1)[~bad], y[~bad], mode, mode)
        _check_e4m3(got.hq[~bad], got.hs.view(8, -1)[~bad], h[~bad], mode, mode)
        groups = (lambda t: t.view(8, 1, cols)) if mode == "row" else (lambda t: t.view(8, -1, 128))
        assert torch.equal(torch.isnan(got.scales.view(8, -1)), torch.isnan(groups(y)).any(-1))
        assert torch.equal(torch.isnan(got.hs.view(8, -1)), (torch.isnan(groups(h)) | torch.isinf(groups(h))).any(-1))
    got = B.loka_add_rmsnorm(x, None, None, 1e-5, out=B.RMS_OUT_MXFP4)
    assert torch.equal(got.scales == 255, torch.isnan(y.view(8, -1, 32)).any(-1))
    # a zero row without eps: 0 / 0 by the formula
    z = B.loka_add_rmsnorm(torch.zeros(2, 128, dtype=torch.bfloat16, device=DEV), None, None, 0.0, out=B.RMS_OUT_BF16)
    assert bool(torch.isnan(z.y).all())


BACK = SHAPES + [(5000, 128), (2100, 1024), (1025, 4096), (530, 8192)]


@pytest.mark.parametrize("gamma,dh", [(True, True), (False, False), (True, False)])
@pytest.mark.parametrize("rows,cols", BACK)
def test_backward(rows, cols, gamma, dh):
    mode = "row" if cols % 128 else ("row", "block", "pow2")[(rows + gamma + dh) % 3]
    x, r, w = _inputs(rows, cols, rows + 7 * cols, gamma=gamma)
    f = B.loka_add_rmsnorm(x, r, w, 1e-5, out=B.RMS_OUT_BF16, ckpt_mode=MODES[mode])
    g = _gen(rows)
    dy = torch.randn(rows, cols, device=DEV, generator=g).bfloat16()
    e = torch.randn(rows, cols, device=DEV, generator=g).bfloat16() if dh else None
    dx, dg = B.loka_rmsnorm_backward(dy, f.hq, f.hs, f.rstd, w, e, ckpt_mode=MODES[mode])
    s = f.hs.double().view(rows, -1)
    h = P.e4m3_values(f.hq) * s.repeat_interleave(cols // s.shape[1], 1)
    want, wdg, mag, dmag = P.rms_backward(dy, h, f.rstd.double().view(-1, 1), w, e)
    # the inner sum adds at most 64 + 6 + 16 terms, with 4 roundings a term; then 4 more on the way out, and bf16
    assert bool(((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + (64 + 6 + 16 + 8) * P.F32 * 2 * mag).all())
    # dgamma: a row after another within a workgroup, then the workgroups
    assert bool(((dg.double() - wdg).abs() <= (rows + 512 + 8) * P.F32 * dmag).all())
    dx2, none = B.loka_rmsnorm_backward(dy, f.hq, f.hs, f.rstd, w, e, ckpt_mode=MODES[mode], want_dgamma=False)
    assert none is None and torch.equal(dx2, dx)
    dx3, dg3 = B.loka_rmsnorm_backward(dy, f.hq, f.hs, f.rstd, w, e, ckpt_mode=MODES[mode])
    assert torch.equal(dx3, dx) and torch.equal(dg3, dg)


def test_a_residual_block_forward_and_backward():
    """norm -> FP8 layer and norm -> 4-bit layer on one residual stream, and back through both to the stream: the calls as a
    trainer makes them, against the plain forms of the same codes."""
    M, D, H = 520, 512, 384
    x, r, w = _inputs(M, D, 77)
    g = _gen(5)
    w1 = (torch.randn(D, H, device=DEV, generator=g) / D ** 0.5).bfloat16()
    up = torch.randn(M, H, device=DEV, generator=g).bfloat16()
    # 8 bits: codes in row scales are the FP8 product's operand
    f = B.loka_add_rmsnorm(x, r, w, ckpt_mode=B.SCALE_BLOCK_1x128)
    wq, sw = B.loka_quantize(w1, B.SCALE_COL, transpose_out=True)
    o, _ = B.loka_fp8_gemm_norm(B.make_desc(M, H, D, norm=B.NORM_NONE), f.y, f.scales, wq, sw)
    a = P.e4m3_values(f.y) * f.scales.double()[:, None]
    b = P.e4m3_values(wq) * sw.double()[:, None]
    # bf16, the sum's roundings, and the FP8 instruction's alignment of 8 products to 2^-13 of the largest
    assert bool(((o.double() - a @ b.t()).abs() <= 2.0 ** -8 * (a @ b.t()).abs() + (7 * 2.0 ** -13 + D / 8 * 2.0 ** -23) * (a.abs() @ b.abs().t())).all())
    # 4 bits
    f4 = B.loka_add_rmsnorm(f.h, None, w, out=B.RMS_OUT_MXFP4, ckpt_mode=B.SCALE_ROW)
    q4, s4 = B.loka_mxfp4_quantize(w1, True)
    o4, _ = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, H, D), f4.y, f4.scales, q4, s4)
    a, b = P.mx_values(f4.y, f4.scales), P.mx_values(q4, s4)
    assert bool(((o4.double() - a @ b.t()).abs() <= 2.0 ** -8 * (a @ b.t()).abs() + (D / 8 + 64) * 2.0 ** -23 * (a.abs() @ b.abs().t())).all())
    # back: through the 4-bit layer to its norm, then on through the 8-bit norm with that gradient arriving past it
    dn, _ = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, D, H), *B.loka_mxfp4_quantize(up), *B.loka_mxfp4_quantize(w1))
    dh, dg4 = B.loka_rmsnorm_backward(dn, f4.hq, f4.hs, f4.rstd, w, ckpt_mode=B.SCALE_ROW)
    dx, dg = B.loka_rmsnorm_backward(dn, f.hq, f.hs, f.rstd, w, dh)
    h4 = P.e4m3_values(f4.hq) * f4.hs.double()[:, None]
    want4, _, mag4, _ = P.rms_backward(dn, h4, f4.rstd.double()[:, None], w, None)
    assert bool(((dh.double() - want4).abs() <= 2.0 ** -8 * want4.abs() + 94 * P.F32 * 2 * mag4).all())
    h8 = P.e4m3_values(f.hq) * f.hs.double().repeat_interleave(128, 1)
    want, wdg, mag, dmag = P.rms_backward(dn, h8, f.rstd.double()[:, None], w, dh)
    assert bool(((dx.double() - want).abs() <= 2.0 ** -8 * want.abs() + 94 * P.F32 * 2 * mag).all())
    assert bool(((dg.double() - wdg).abs() <= (M + 520) * P.F32 * dmag).all()) and dg4.shape == (D,)


def test_gradient_against_differences():
    # d/dt sum(up * y(x + t v)) by central differences of the 64-bit forward at the checkpoint's values, against <dx, v>
    rows, cols = 6, 256
    x, _, w = _inputs(rows, cols, 3, residual=False)
    f = B.loka_add_rmsnorm(x, None, w, out=B.RMS_OUT_BF16, ckpt_mode=B.SCALE_ROW)
    h = P.e4m3_values(f.hq) * f.hs.double()[:, None]
    rstd = (1 / torch.sqrt((h * h).mean(1) + 1e-5))
    up, v = (torch.randn(rows, cols, device=DEV, generator=_gen(i)).bfloat16() for i in (1, 2))
    dx, dg = B.loka_rmsnorm_backward(up, f.hq, f.hs, rstd.float(), w, ckpt_mode=B.SCALE_ROW)
    t = 1e-4
    loss = lambda hh, ww: (up.double() * P.rms_forward(hh, None, ww, 1e-5)[2]).sum(1)
    diff = (loss(h + t * v.double(), w) - loss(h - t * v.double(), w)) / (2 * t)
    # bf16 rounding of dx, and the differences' own t^2 and 1e-16 / t
    tol = 2.0 ** -8 * (dx.double().abs() * v.double().abs()).sum(1) + 1e-5 * diff.abs() + 1e-5
    assert bool(((dx.double() * v.double()).sum(1) - diff).abs().le(tol).all())
    u = torch.randn(cols, device=DEV, generator=_gen(4)).double()
    dgd = (loss(h, w.double() + t * u).sum() - loss(h, w.double() - t * u).sum()) / (2 * t)
    assert abs(float((dg.double() * u).sum() - dgd)) <= 1e-5 * float((dg.double() * u).abs().sum())


@pytest.mark.parametrize("cols", [128, 256, 496, 1008, 2048, 4096, 8192, 16384, 32768])
def test_rows_that_pass_the_caches_by(cols):
    # a call of 2^26 elements and more, against its halves
    rows = (1 << 26) // cols + 3
    x, r, w = _inputs(rows, cols, cols)
    blk = B.SCALE_BLOCK_1x128 if cols % 128 == 0 else B.SCALE_ROW
    parts = slice(0, rows // 2), slice(rows // 2, rows)
    for out in (B.RMS_OUT_BF16, B.RMS_OUT_MXFP4):
        kw = dict(out=out, ckpt_mode=blk)
        f, halves = B.loka_add_rmsnorm(x, r, w, **kw), [B.loka_add_rmsnorm(x[p], r[p], w, **kw) for p in parts]
        for k in ("h", "y", "hq", "hs", "rstd") + (("scales",) if out != B.RMS_OUT_BF16 else ()):
            for p, h in zip(parts, halves):
                assert torch.equal(getattr(f, k)[p], getattr(h, k)), k
    dx, dg = B.loka_rmsnorm_backward(r, f.hq, f.hs, f.rstd, w, x, ckpt_mode=blk)
    sums = 0
    for p, h in zip(parts, halves):
        part, part_dg = B.loka_rmsnorm_backward(r[p], h.hq, h.hs, h.rstd, w, x[p], ckpt_mode=blk)
        assert torch.equal(dx[p], part)
        sums = sums + part_dg.double()
    # a column's terms in chains of rows / 512, 16 rows of a workgroup, 16 and 32 partial sums; two such sums, each term with 3 roundings
    values = P.e4m3_values(f.hq).view(rows, cols).abs()
    scale = f.hs.double().view(rows, -1, 1) * f.rstd.double().view(rows, 1, 1)
    size = ((values.view(rows, f.hs.numel() // rows, -1) * scale).view(rows, cols) * r.double().abs()).sum(0)
    assert bool(((dg.double() - sums).abs() <= 2 * (rows / 512 + 1 + 64 + 3) * P.F32 * size).all())


def test_rows_past_4_gb():
    rows, cols = (1 << 20) + 19, 4224                 # codes and bf16 rows beyond 2^32 bytes
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    tail, _, w = _inputs(64, cols, 9, residual=False)
    x[-64:] = tail
    kw = dict(out_mode=B.SCALE_BLOCK_1x128, ckpt_mode=B.SCALE_BLOCK_1x128)
    a, b = B.loka_add_rmsnorm(x, None, w, **kw), B.loka_add_rmsnorm(tail, None, w, **kw)
    assert torch.equal(a.y[-64:], b.y) and torch.equal(a.hq[-64:], b.hq) and torch.equal(a.hs[-64:], b.hs) and not bool(a.y[:-64].any())
    dx, dg = B.loka_rmsnorm_backward(x, a.hq, a.hs, a.rstd, w, x)
    dx2, dg2 = B.loka_rmsnorm_backward(tail, b.hq, b.hs, b.rstd, w, tail)
    assert torch.equal(dx[-64:], dx2) and not bool(dx[:-64].any())
    assert bool(((dg - dg2).double().abs() <= 2 * 600 * P.F32 * (tail.double() * tail.double() * b.rstd.double()[:, None]).abs().sum(0) * 1.1).all())


def test_replays_from_a_graph_and_runs_on_another_stream():
    rows, cols = 600, 1024
    x, r, w = _inputs(rows, cols, 1)

    def step():
        f = B.loka_add_rmsnorm(x, r, w, ckpt_mode=B.SCALE_BLOCK_1x128)
        dx, dg = B.loka_rmsnorm_backward(r, f.hq, f.hs, f.rstd, w, x)
        return f.h, f.y, f.scales, f.hq, f.hs, f.rstd, dx, dg

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kept = step()
    for seed in (2, 3, 4):
        x.normal_(generator=_gen(seed))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = step()
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(other, eager))
