"""Every kernel form of the MXFP4 product, on operands whose sums are exact in fp32 in any order: values are compared for equality."""
import ctypes

import pytest
import torch

import mxfp4_shapes as S
import plain_ops as P
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _operand(rows, K, seed, codes=16, scales=(127, 128)):
    """Stored operand of random codes and scale bytes: each group with a scale of its own, zeros past K."""
    kp, g = P.padded(K), _gen(seed)
    c = torch.randint(0, 16, (rows, kp), device=DEV, generator=g, dtype=torch.uint8)
    if codes < 16:                     # magnitudes of the first codes only
        c = (c & 8) | (c & 7) % codes
    c[:, K:] = 0
    s = torch.tensor(scales, dtype=torch.uint8, device=DEV)[torch.randint(0, len(scales), (rows, kp // 32), device=DEV, generator=g)]
    s[:, -(-K // 32):] = 0
    return c[:, 0::2] | c[:, 1::2] << 4, s


def _exact(xq, sx, wq, sw):
    """The products' sums.  Every product is a multiple of 1/4, and all of them together stay below 2^24 such units, so each partial sum
    in any order is a number that fp32 holds."""
    a, b = P.mx_values(xq, sx), P.mx_values(wq, sw)
    assert float((torch.nan_to_num(a).abs() @ torch.nan_to_num(b).abs().t()).max()) * 4 < 2 ** 24
    return a @ b.t()


def _problem(t, g, batch):
    return t.view(batch, -1, t.shape[-1])[g]


@pytest.mark.parametrize("form,M,N,K,batch", S.ALL)
def test_products_of_each_form(form, M, N, K, batch):
    xq, sx = _operand(batch * M, K, 1)
    wq, sw = _operand(batch * N, K, 2)
    want = torch.cat([_exact(*(_problem(t, g, batch) for t in (xq, sx, wq, sw))) for g in range(batch)]).float()
    d = B.make_mxfp4_desc(M, N, K, batch)
    out, y = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True)
    assert torch.equal(y, want) and torch.equal(out, want.bfloat16())
    assert torch.equal(B.loka_mxfp4_gemm(d, xq, sx, wq, sw)[0], want.bfloat16())
    assert torch.equal(B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_out=False, want_y=True)[1], want)


@pytest.mark.parametrize("M,N,K,batch", S.SHAPES[S.SPLIT])
def test_the_workspace_of_a_split_contraction(M, N, K, batch):
    xq, sx = _operand(batch * M, K, 3)
    wq, sw = _operand(batch * N, K, 4)
    want = torch.cat([_exact(*(_problem(t, g, batch) for t in (xq, sx, wq, sw))) for g in range(batch)]).float()
    d = B.make_mxfp4_desc(M, N, K, batch)
    need = B.lib().loka_mxfp4_gemm_workspace(ctypes.byref(d))
    assert need > 0
    # NaNs in it do not matter, nothing behind it is written; less than it asks for: unsplit, and nothing of it is written
    for room, used in ((need, True), (need + 64, True), (need - 1, False), (16, False), (0, False)):
        ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
        out, y = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True, workspace=ws[:room])
        assert torch.equal(y, want) and torch.equal(out, want.bfloat16()), room
        assert bool((ws[need if used else 0:] == 0xFF).all()), room
    d.strideO = M * N + 5              # problems apart from each other: what lies between them stays
    span = (batch - 1) * d.strideO + M * N
    out, y = torch.full((span,), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((span,), 7.0, device=DEV)
    B.loka_mxfp4_gemm(d, xq, sx, wq, sw, out=out, y=y)
    for g in range(batch):
        at = slice(g * d.strideO, g * d.strideO + M * N)
        assert torch.equal(y[at].view(M, N), want[g * M:(g + 1) * M]) and torch.equal(out[at].view(M, N), want[g * M:(g + 1) * M].bfloat16())
        assert bool((y[at.stop: at.stop + 5] == 7).all()) and bool((out[at.stop: at.stop + 5] == 7).all())


@pytest.mark.parametrize("shared", ["x", "w", "both", "gaps"])
@pytest.mark.parametrize("form,M,N,K,batch", [s for s in S.ALL if s[4] > 1])
def test_shared_operands_and_operands_apart(form, M, N, K, batch, shared):
    one_x, one_w, gap = shared in ("x", "both"), shared in ("w", "both"), shared == "gaps"
    d = B.make_mxfp4_desc(M, N, K, batch)
    kp = P.padded(K)
    # rows between the problems hold NaN groups, which must reach nothing
    more_x, more_w = (3, 5) if gap else (0, 0)
    xq, sx = _operand((1 if one_x else batch) * (M + more_x), K, 5)
    wq, sw = _operand((1 if one_w else batch) * (N + more_w), K, 6)
    d.strideX, d.strideW = 0 if one_x else (M + more_x) * kp, 0 if one_w else (N + more_w) * kp
    if gap:
        sx.view(batch, M + more_x, -1)[:, M:] = 255
        sw.view(batch, N + more_w, -1)[:, N:] = 255
    out, y = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True)
    for g in range(batch):
        x = [_problem(t, 0 if one_x else g, 1 if one_x else batch)[:M] for t in (xq, sx)]
        w = [_problem(t, 0 if one_w else g, 1 if one_w else batch)[:N] for t in (wq, sw)]
        want = _exact(*x, *w).float()
        assert torch.equal(y[g * M:(g + 1) * M], want) and torch.equal(out[g * M:(g + 1) * M], want.bfloat16()), g


@pytest.mark.parametrize("form,M,N,K,batch", [s for s in S.ALL if s[4] == 1])
def test_one_product_at_every_place(form, M, N, K, batch):
    # one nonzero in each row on each side, at changing places, with scales of its own: every result is that product or nothing
    kp, m, n = P.padded(K), torch.arange(M, device=DEV), torch.arange(N, device=DEV)
    xq, wq = (torch.zeros(r, kp // 2, dtype=torch.uint8, device=DEV) for r in (M, N))
    sx = (120 + torch.arange(M * (kp // 32), device=DEV) % 13).to(torch.uint8).view(M, -1)
    sw = (121 + torch.arange(N * (kp // 32), device=DEV) % 11).to(torch.uint8).view(N, -1)
    kx, kw = m * 7 % K, n * 3 % K
    xq[m, kx // 2] = ((m % 15 + 1) << (4 * (kx % 2))).to(torch.uint8)
    wq[n, kw // 2] = ((n % 13 + 1) << (4 * (kw % 2))).to(torch.uint8)
    _, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K), xq, sx, wq, sw, want_y=True)
    a, b = P.mx_values(xq, sx)[m, kx], P.mx_values(wq, sw)[n, kw]
    assert torch.equal(y.double(), torch.where(kx[:, None] == kw[None], a[:, None] * b[None], 0.0))


@pytest.mark.parametrize("form,M,N,K,batch", S.ALL)
def test_nan_groups_reach_their_rows_and_columns_only(form, M, N, K, batch):
    xq, sx = _operand(batch * M, K, 7)
    wq, sw = _operand(batch * N, K, 8)
    groups = -(-K // 32)
    for t, s, rows in ((xq, sx, (0, M // 2, batch * M - 1)), (wq, sw, (1, N // 2 + 1, batch * N - 2))):
        for i, r in enumerate(rows):   # first, some and last group
            k = (0, groups // 2, groups - 1)[i]
            s[r, k] = 255
            t[r, k * 16:(k + 1) * 16] = 0
    want = torch.cat([_exact(*(_problem(t, g, batch) for t in (xq, sx, wq, sw))) for g in range(batch)]).float()
    assert bool(torch.isnan(want).any()) and not bool(torch.isnan(want).all())
    out, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K, batch), xq, sx, wq, sw, want_y=True)
    for got, ref in ((y, want), (out, want.bfloat16())):
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(ref))


@pytest.mark.parametrize("M,N,K", [(1, 40, 100000), (5, 3, 100000), (64, 100, 70000), (129, 130, 100032)])
def test_no_element_of_a_long_contraction_is_lost(M, N, K):
    xq, sx = _operand(M, K, 9, codes=3, scales=(127,))
    wq, sw = _operand(N, K, 10, codes=3, scales=(127,))
    d = B.make_mxfp4_desc(M, N, K)
    want = _exact(xq, sx, wq, sw).float()
    out, y = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True)
    assert torch.equal(y, want) and torch.equal(out, want.bfloat16())
    x = P.mx_values(xq, sx)[:, :K].bfloat16()       # (its own codes have other scales, and stand for the same values)
    out, y = B.loka_mxfp4_linear(d, x, wq, sw, want_y=True)
    assert torch.equal(y, want) and torch.equal(out, want.bfloat16())


LAYERS = [s for s in S.ALL if s[4] == 1]


@pytest.mark.parametrize("form,M,N,K,batch", LAYERS)
def test_the_layer_is_the_quantization_and_the_product(form, M, N, K, batch):
    x = torch.randn(M, K, device=DEV, generator=_gen(M)).bfloat16()
    wq, sw = _operand(N, K, 11)
    d = B.make_mxfp4_desc(M, N, K)
    out, y = B.loka_mxfp4_linear(d, x, wq, sw, want_y=True)
    if M > 16:
        o2, y2 = B.loka_mxfp4_gemm(d, *B.loka_mxfp4_quantize(x), wq, sw, want_y=True)
        assert torch.equal(y, y2) and torch.equal(out, o2)
    a, b = P.mx_values(*P.mx_quantize(x)), P.mx_values(wq, sw)
    # fp32: at most one addition per 8 products and per partial sum, each off by at most a step
    assert bool(((y.double() - a @ b.t()).abs() <= (K / 8 + 64) * 2.0 ** -23 * (a.abs() @ b.abs().t())).all())


def test_each_form_from_a_graph_and_on_two_streams():
    work = []
    for form, M, N, K, _ in (LAYERS[0], *(next(s for s in LAYERS if s[0] == f) for f in (S.LARGE, S.HALVES, S.SMALL, S.SPLIT))):
        work.append((B.make_mxfp4_desc(M, N, K), torch.empty(M, K, dtype=torch.bfloat16, device=DEV), *_operand(N, K, N)))
    assert {B.lib().loka_test_mxfp4_form(ctypes.byref(w[0])) for w in work} == {S.STREAM, S.LARGE, S.HALVES, S.SMALL}

    def step():
        got = []
        for d, x, wq, sw in work:
            got += B.loka_mxfp4_linear(d, x, wq, sw, want_y=True)
            got += B.loka_mxfp4_gemm(d, *B.loka_mxfp4_quantize(x), wq, sw, want_y=True)
        return got

    def fill(seed):
        for i, w in enumerate(work):
            w[1].normal_(generator=_gen(seed + i))

    fill(0)
    step()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kept = step()
    for seed in (10, 20, 30):
        fill(seed)
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, eager))
        for t in kept:
            t.zero_()
        torch.cuda.synchronize()
        both = []
        for s in (side, other):        # two at once, and the graph behind them
            with torch.cuda.stream(s):
                both.append(step())
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        for got in (*both, kept):
            assert all(torch.equal(a, b) for a, b in zip(got, eager))


def test_columns_quantized_past_4_gb():
    M, K = (1 << 21) + 37, 4096        # (32 rows a group: the last group has 5)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    first = (M - 300) // 32 * 32
    x[first:] = torch.randn(M - first, K, device=DEV, generator=_gen(12)).bfloat16()
    x[:64] = torch.randn(64, K, device=DEV, generator=_gen(13)).bfloat16()
    q, s = B.loka_mxfp4_quantize(x, True)
    for a, b in ((0, 64), (first, M)):
        wq, ws = P.mx_quantize(x[a:b].t())
        n = -(-(b - a) // 32)
        assert torch.equal(q[:, a // 2: a // 2 + n * 16], wq[:, : n * 16]) and torch.equal(s[:, a // 32: a // 32 + n], ws[:, :n])
    assert not bool(q[:, 32: first // 2].any()) and not bool(s[:, 2: first // 32].any())
    end = -(-M // 32)
    assert not bool(q[:, end * 16:].any()) and not bool(s[:, end:].any())


def test_every_scale_byte():
    # values of all codes under all bytes (those beyond bf16's range are infinite, 255 is NaN), and the product of every pair of scales
    byte = torch.arange(256, device=DEV, dtype=torch.uint8)
    q = torch.zeros(256, 64, dtype=torch.uint8, device=DEV)
    q[:, :8] = torch.tensor([0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE], dtype=torch.uint8, device=DEV)
    s = byte[:, None].repeat(1, 4).contiguous()
    got, want = B.loka_mxfp4_dequantize(q, s, 16).double(), P.mx_values(q, s)[:, :16].float().bfloat16().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))
    for M, N, form in ((255, 255, S.STREAM), (4080, 4080, S.SMALL)):
        d = B.make_mxfp4_desc(M, N, 128)
        assert B.lib().loka_test_mxfp4_form(ctypes.byref(d)) == form
        (xq, sx), (wq, sw) = ((torch.zeros(r, 64, dtype=torch.uint8, device=DEV), torch.zeros(r, 4, dtype=torch.uint8, device=DEV)) for r in (M, N))
        xq[:, 0], wq[:, 0] = 2, 2
        sx[:, 0], sw[:, 0] = byte[torch.arange(M, device=DEV) % 255], byte[torch.arange(N, device=DEV) % 255]
        _, y = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True)
        # a power of two: exact down to the last subnormal, 0 below, infinite from 2^128 on
        assert torch.equal(y, (P.mx_values(xq, sx)[:, :1] * P.mx_values(wq, sw)[:, :1].t()).float())
