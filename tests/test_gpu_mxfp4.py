"""MXFP4 quantization and products against plain 64-bit forms: codes and scales bit for bit, products within the rounding of
their fp32 sums."""
import ctypes

import pytest
import torch

import plain_ops as P
from paper_2605_10886_amd import binding as B
from paper_2605_10886_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _wide(rows, cols, seed):
    """Values of every magnitude that the format meets: exponents spread over the groups, zeros, values between two codes."""
    g = _gen(seed)
    x = torch.randn(rows, cols, device=DEV, generator=g) * torch.exp2(torch.randint(-30, 30, (rows, 1), device=DEV, generator=g).float())
    x *= torch.exp2(torch.randint(-4, 1, (rows, cols), device=DEV, generator=g).float())
    x[torch.rand(rows, cols, device=DEV, generator=g) < 0.05] = 0.0
    return x.bfloat16()


def _same(got, want):
    assert got.shape == want.shape and torch.equal(got, want), f"{int((got != want).sum())} of {want.numel()} differ"


SHAPES = [(1, 1), (1, 32), (3, 31), (2, 33), (5, 128), (7, 127), (16, 129), (17, 720), (130, 1008), (33, 2049), (300, 384), (1, 70000)]


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_codes_and_values(shape, transpose):
    x = _wide(*shape, seed=sum(shape))
    q, s = B.loka_mxfp4_quantize(x, transpose)
    t = x.t() if transpose else x
    wq, ws = P.mx_quantize(t)
    _same(q, wq)
    _same(s, ws)
    v = B.loka_mxfp4_dequantize(q, s, t.shape[1])
    assert torch.equal(v.double(), P.mx_values(wq, ws)[:, :t.shape[1]])


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("ld,offset", [(104, 0), (103, 0), (104, 1), (104, 2), (128, 8)])
def test_strides_and_alignment(ld, offset, transpose):
    buf = _wide(1, 41 * ld + 16, seed=ld + offset).view(-1)
    x = buf[offset:].as_strided((40, 90), (ld, 1), offset)
    q, s = B.loka_mxfp4_quantize(x, transpose)
    wq, ws = P.mx_quantize((x.t() if transpose else x).contiguous())
    _same(q, wq)
    _same(s, ws)
    if not transpose:                  # values into rows of a larger matrix, the rest of which stays
        out = torch.full((40, ld), 7.0, dtype=torch.bfloat16, device=DEV)
        B.loka_mxfp4_dequantize(q, s, 90, out=out[:, :90])
        assert torch.equal(out[:, :90].double(), P.mx_values(wq, ws)[:, :90]) and bool((out[:, 90:] == 7).all())


@pytest.mark.parametrize("rows,cols", [(1, 7), (9, 1), (5, 33), (300, 31), (257, 1003), (1008, 5013), (3, 70001)])
def test_values_of_rows_that_start_anywhere(rows, cols):
    x = _wide(rows, cols, seed=rows)
    x[rows // 2, cols // 2] = float("nan")
    q, s = B.loka_mxfp4_quantize(x)
    want = P.mx_values(q, s)[:, :cols]
    for out in (None, torch.empty(rows * cols + 1, dtype=torch.bfloat16, device=DEV)[1:].view(rows, cols)):      # aligned or not
        v = B.loka_mxfp4_dequantize(q, s, cols, out=out).double()
        assert torch.equal(torch.isnan(v), torch.isnan(want)) and torch.equal(torch.nan_to_num(v), torch.nan_to_num(want))


def test_every_bf16_value_ties_and_special_groups():
    # every finite bf16 with every group maximum from its own exponent up to three above, and the halves between codes
    allb = torch.arange(65536, device=DEV, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    allb = allb[torch.isfinite(allb)]
    for up in (1.0, 2.0, 4.0, 7.0):
        x = torch.zeros(allb.numel(), 32, dtype=torch.bfloat16, device=DEV)
        x[:, 3] = allb
        x[:, 9] = (allb.float() * up).bfloat16()
        x[~torch.isfinite(x).all(1)] = 1.0
        q, s = B.loka_mxfp4_quantize(x)
        wq, ws = P.mx_quantize(x)
        _same(q, wq)
        _same(s, ws)
        assert torch.equal(B.loka_mxfp4_dequantize(q, s, 32).double(), P.mx_values(wq, ws)[:, :32])
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -0.0], device=DEV)
    x = torch.cat([ties, torch.full((16,), 4.0, device=DEV)]).repeat(4, 1).bfloat16() * torch.tensor([[1.0], [2.0 ** -100], [2.0 ** 100], [2.0 ** -126]], device=DEV).bfloat16()
    q, s = B.loka_mxfp4_quantize(x)
    wq, ws = P.mx_quantize(x)
    _same(q, wq)
    _same(s, ws)
    # a NaN or an infinity takes its group and no other
    x = _wide(4, 256, seed=5)
    x[0, 40], x[1, 0], x[2, 255] = float("nan"), float("inf"), float("-inf")
    for tr in (False, True):
        q, s = B.loka_mxfp4_quantize(x, tr)
        t = x.t() if tr else x
        wq, ws = P.mx_quantize(t)
        _same(q, wq)
        _same(s, ws)
        v = B.loka_mxfp4_dequantize(q, s, t.shape[1])
        want = P.mx_values(wq, ws)[:, :t.shape[1]]
        assert torch.equal(torch.isnan(v), torch.isnan(want)) and torch.equal(torch.nan_to_num(v.double()), torch.nan_to_num(want))


def _operand(rows, K, seed, scale=1.0):
    x = (torch.randn(rows, K, device=DEV, generator=_gen(seed)) * scale).bfloat16()
    return (x, *B.loka_mxfp4_quantize(x))


def _check(y, xq, sx, wq, sw, K, out=None):
    """fp32 y within the rounding of its sum: the products are exact, at most one fp32 addition per 8 of them and per partial
    sum, each off by at most a step (2^-23: the order and the rounding of the instruction's own additions are not specified)."""
    a, b = P.mx_values(xq, sx), P.mx_values(wq, sw)
    ref, mag = a @ b.t(), a.abs() @ b.abs().t()
    tol = (P.padded(K) / 8 + 64) * 2.0 ** -23 * mag
    assert bool((y.double() - ref).abs().le(tol).all()), float(((y.double() - ref).abs() / tol.clamp_min(1e-300)).max())
    if out is not None:
        assert torch.equal(out, y.bfloat16())


PRODUCTS = [(1, 1, 1), (1, 16, 128), (2, 17, 33), (1, 4096, 4096), (3, 1000, 1111), (13, 64, 8192), (16, 520, 512), (16, 48, 640), (17, 40, 200),
            (33, 65, 1030), (64, 256, 256), (100, 100, 100), (129, 257, 384), (127, 255, 4096), (256, 256, 512), (300, 720, 1008),
            (513, 1030, 640), (260, 516, 16384), (64, 100, 70000), (1024, 768, 256), (5, 3, 100000), (2500, 130, 64),
            # several result tiles a workgroup, in each form of the tile kernel
            (6000, 6000, 2000), (6001, 6003, 2000), (8200, 8200, 300), (4104, 4104, 4160), (20000, 72, 130)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_products(M, N, K):
    x, xq, sx = _operand(M, K, 1)
    _, wq, sw = _operand(N, K, 2, K ** -0.5)
    d = B.make_mxfp4_desc(M, N, K)
    out, y = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True)
    _check(y, xq, sx, wq, sw, K, out)
    o2, none = B.loka_mxfp4_gemm(d, xq, sx, wq, sw)
    none2, y2 = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_out=False, want_y=True)
    assert none is None and none2 is None and torch.equal(o2, out) and torch.equal(y2, y)
    # the layer quantizes x as loka_mxfp4_quantize does; its sums may be in another order
    lo, ly = B.loka_mxfp4_linear(d, x, wq, sw, want_y=True)
    _check(ly, xq, sx, wq, sw, K, lo)
    lo2, _ = B.loka_mxfp4_linear(d, x, wq, sw)
    assert torch.equal(lo, lo2)
    # without room for partial sums
    none = torch.empty(0, dtype=torch.uint8, device=DEV)
    o3, y3 = B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_y=True, workspace=none)
    _check(y3, xq, sx, wq, sw, K, o3)


def test_each_code_and_scale_reaches_its_place():
    # one nonzero per row on each side, at every place of a stored row, with a scale of its own: Y is that product alone
    K = 640
    k = torch.arange(K, device=DEV)
    for M, N in ((8, K), (16, K), (K, 16), (K, K)):
        xq = torch.zeros(M, K // 2, dtype=torch.uint8, device=DEV)
        wq = torch.zeros(N, K // 2, dtype=torch.uint8, device=DEV)
        sx = (120 + torch.arange(M * (K // 32), device=DEV) % 13).to(torch.uint8).view(M, -1)
        sw = (121 + torch.arange(N * (K // 32), device=DEV) % 11).to(torch.uint8).view(N, -1)
        kx, kw = k[:M] * 7 % K if M < K else k, k[:N] * 3 % K if N < K else k
        cx, cw = torch.arange(M, device=DEV) % 15 + 1, torch.arange(N, device=DEV) % 13 + 1
        xq[torch.arange(M, device=DEV), kx // 2] = (cx << (4 * (kx % 2))).to(torch.uint8)
        wq[torch.arange(N, device=DEV), kw // 2] = (cw << (4 * (kw % 2))).to(torch.uint8)
        _, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K), xq, sx, wq, sw, want_y=True)
        assert torch.equal(y.double(), P.mx_values(xq, sx) @ P.mx_values(wq, sw).t())


@pytest.mark.parametrize("M", [2, 16, 200])
def test_nan_groups_reach_their_rows_and_columns_only(M):
    K, N = 512, 192
    x = torch.randn(M, K, device=DEV, generator=_gen(3)).bfloat16()
    w = torch.randn(N, K, device=DEV, generator=_gen(4)).bfloat16()
    x[1, 77], w[5, 500] = float("inf"), float("nan")
    wq, sw = B.loka_mxfp4_quantize(w)
    out, _ = B.loka_mxfp4_linear(B.make_mxfp4_desc(M, N, K), x, wq, sw)
    want = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    want[1], want[:, 5] = True, True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("M,N,K,G,shared", [(4, 40, 96, 3, False), (33, 130, 200, 5, True), (300, 256, 256, 4, False), (16, 16, 1000, 7, True)])
def test_grouped(M, N, K, G, shared):
    _, xq, sx = _operand(G * M, K, 5)
    _, wq, sw = _operand(N if shared else G * N, K, 6)
    out, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K, G, shared_w=shared), xq, sx, wq, sw, want_y=True)
    for g in range(G):
        r, c = slice(g * M, g * M + M), slice(0, N) if shared else slice(g * N, g * N + N)
        _check(y[r], xq[r], sx[r], wq[c], sw[c], K, out[r])
    # problems apart from each other, and one X for all
    for gap in (8, 3):
        d = B.make_mxfp4_desc(M, N, K, G, shared_w=shared)
        d.strideO = M * N + gap
        far = torch.full((G * d.strideO,), 3.0, device=DEV)
        d.strideX = 0
        B.loka_mxfp4_gemm(d, xq, sx, wq, sw, want_out=False, y=far)
        for g in range(G):
            c = slice(0, N) if shared else slice(g * N, g * N + N)
            part = far[g * d.strideO:(g + 1) * d.strideO]
            _check(part[:M * N].view(M, N), xq[:M], sx[:M], wq[c], sw[c], K)
            assert bool((part[M * N:] == 3).all())


@pytest.mark.parametrize("M", [1, 2, 3, 9, 16, 17, 70])
@pytest.mark.parametrize("K,ld,offset", [(1000, 1008, 8), (1000, 1007, 0), (1000, 1000, 1), (999, 1000, 0), (4736, 5000, 16)])
def test_layer_on_rows_of_a_larger_matrix(M, K, ld, offset):
    N = 80
    buf = torch.randn((M + 1) * ld + 64, device=DEV, generator=_gen(M)).bfloat16()
    x = buf.as_strided((M, K), (ld, 1), offset)
    _, wq, sw = _operand(N, K, 8, K ** -0.5)
    out, y = B.loka_mxfp4_linear(B.make_mxfp4_desc(M, N, K), x, wq, sw, want_y=True)
    _check(y, *P.mx_quantize(x.contiguous()), wq, sw, K, out)


@pytest.mark.parametrize("M", [1, 2, 3, 11, 16])
@pytest.mark.parametrize("K,N", [(5, 4100), (7, 33), (8, 4100), (9, 20), (515, 4100), (513, 8200), (1031, 16400), (1024, 4112), (1024, 8208), (2056, 16400)])
def test_layer_on_few_rows_of_many_columns(M, K, N):
    x = _wide(1, M * K, seed=K).view(M, K)
    _, wq, sw = _operand(N, K, 8, K ** -0.5)
    out, y = B.loka_mxfp4_linear(B.make_mxfp4_desc(M, N, K), x, wq, sw, want_y=True)
    stored = P.mx_quantize(x)
    _check(y, *stored, wq, sw, K, out)
    out, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K), *stored, wq, sw, want_y=True)
    _check(y, *stored, wq, sw, K, out)


def test_two_streams_at_once():
    shapes = [(16, 2048, 4096), (300, 1024, 2048), (64, 512, 512), (2000, 512, 1024)]
    work = [(B.make_mxfp4_desc(M, N, K), torch.randn(M, K, device=DEV, generator=_gen(M)).bfloat16(), *_operand(N, K, N)[1:]) for M, N, K in shapes]
    want = [B.loka_mxfp4_linear(*w)[0] for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(5):
        for i, w in enumerate(work):
            with torch.cuda.stream(streams[i % 2]):
                got.append((i, B.loka_mxfp4_linear(*w)[0]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i, o in got)


@pytest.mark.parametrize("M,K,N", [(50, 33, 70), (700, 256, 320), (5013, 128, 96)])
def test_training_step(M, K, N):
    # forward, dX = dY W^T and dW = X^T dY, each operand quantized along its contraction
    g = _gen(9)
    x, w, dy = (torch.randn(s, device=DEV, generator=g).bfloat16() for s in ((M, K), (K, N), (M, N)))
    for (mk, mn, ml), a, b in (((M, N, K), B.loka_mxfp4_quantize(x), B.loka_mxfp4_quantize(w, True)),
                               ((M, K, N), B.loka_mxfp4_quantize(dy), B.loka_mxfp4_quantize(w)),
                               ((K, N, M), B.loka_mxfp4_quantize(x, True), B.loka_mxfp4_quantize(dy, True))):
        out, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(mk, mn, ml), *a, *b, want_y=True)
        _check(y, *a, *b, ml, out)


@pytest.mark.parametrize("K", [4104, 4103])
def test_values_that_pass_the_caches_by(K):
    # inputs and results of 2^27 elements and more: codes against those of the halves, small whole numbers against exact products
    M = 32768 + 131
    x = _wide(1, M * K, seed=3).view(M, K)
    q, s = B.loka_mxfp4_quantize(x)
    qt, st = B.loka_mxfp4_quantize(x, True)
    for a, b in ((0, 16384), (16384, M)):
        hq, hs = B.loka_mxfp4_quantize(x[a:b])
        _same(q[a:b], hq)
        _same(s[a:b], hs)
        hq, hs = B.loka_mxfp4_quantize(x[a:b], True)
        _same(qt[:, a // 2: a // 2 + hq.shape[1]], hq)
        _same(st[:, a // 32: a // 32 + hs.shape[1]], hs)
    del x, q, s, qt, st
    K, N = 160, K
    codes = torch.tensor([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    x, w = (codes[torch.randint(0, 15, s, device=DEV, generator=_gen(s[0]))].bfloat16() for s in ((M, K), (N, K)))
    x[:, ::32], w[:, ::32] = 6, 6      # (every group's scale is 1)
    a, b = B.loka_mxfp4_quantize(x), B.loka_mxfp4_quantize(w)
    want = (x.float() @ w.float().t()).bfloat16()      # multiples of 1/4 up to 5760: exact in fp32
    d = B.make_mxfp4_desc(M, N, K)
    out, _ = B.loka_mxfp4_gemm(d, *a, *b)
    _same(out, want)
    out, _ = B.loka_mxfp4_linear(d, x, *b)
    _same(out, want)
    out, y = B.loka_mxfp4_gemm(d, *a, *b, want_y=True)
    _same(out, want)
    _same(y.bfloat16(), want)


@pytest.mark.parametrize("batch,M,N,K", [(b, M, N, 100) for b in (1, 3) for M in (17, 300, 1025) for N in (1, 7, 13, 250, 257, 1001, 4098)] +
                         [(1, 20000, 515, 100), (9, 3000, 258, 70), (1, 4096, 4095, 512), (1, 4200, 4098, 512), (3, 2111, 4033, 300), (2, 70001, 129, 100)])
def test_results_whose_rows_start_anywhere(batch, M, N, K):
    # small whole numbers: exact sums; results side by side, so that a value written past its row or problem shows
    codes = torch.tensor([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    x, w = (codes[torch.randint(0, 15, s, device=DEV, generator=_gen(s[1]))].bfloat16() for s in ((batch * M, K), (batch * N, K)))
    x[:, ::32], w[:, ::32] = 6, 6
    d = B.make_mxfp4_desc(M, N, K, batch)
    d.strideO = M * N + 5              # (the values between the problems stay)
    span = (batch - 1) * d.strideO + M * N
    out, y = torch.full((span,), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((span,), 7.0, device=DEV)
    B.loka_mxfp4_gemm(d, *B.loka_mxfp4_quantize(x), *B.loka_mxfp4_quantize(w), out=out, y=y)
    want = torch.full((span,), 7.0, device=DEV)
    for b in range(batch):
        want[b * d.strideO: b * d.strideO + M * N] = (x[b * M: (b + 1) * M].float() @ w[b * N: (b + 1) * N].float().t()).flatten()
    _same(y, want)
    _same(out, want.bfloat16())


def test_rows_past_4_gb():
    # stored codes beyond 2^32 bytes: the last rows of a tall operand, against the same rows alone
    M, K, N = (1 << 21) + 37, 4096, 32
    xq = torch.zeros(M, K // 2, dtype=torch.uint8, device=DEV)
    sx = torch.full((M, K // 32), 127, dtype=torch.uint8, device=DEV)
    _, tq, ts = _operand(300, K, 11)
    xq[-300:], sx[-300:] = tq, ts
    _, wq, sw = _operand(N, K, 12)
    out, _ = B.loka_mxfp4_gemm(B.make_mxfp4_desc(M, N, K), xq, sx, wq, sw)
    a, b = P.mx_values(tq, ts), P.mx_values(wq, sw)
    tol = (K / 8 + 64) * 2.0 ** -23 * (a.abs() @ b.abs().t()) + 2.0 ** -8 * (a @ b.t()).abs()
    assert bool((out[-300:].double() - a @ b.t()).abs().le(tol).all()) and not bool(out[:-300].any())
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV)
    x[-300:] = B.loka_mxfp4_dequantize(tq, ts, K)
    q, s = B.loka_mxfp4_quantize(x)
    assert torch.equal(B.loka_mxfp4_dequantize(q[-300:], s[-300:], K), x[-300:]) and not bool(q[:-300].any())
    del q, s
    q, s = B.loka_mxfp4_quantize(x, True)
    assert not bool(q[:, : (M - 300) // 256 * 128].any())
    assert torch.equal(B.loka_mxfp4_dequantize(q, s, M)[:, -300:].t().abs().amax(), x[-300:].abs().amax())


def test_replays_from_a_graph_and_runs_on_another_stream():
    M, K, N = 300, 1008, 512
    _, wq, sw = _operand(N, K, 21)
    _, w8, s8 = _operand(N, K, 22)
    x = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    d, d1 = B.make_mxfp4_desc(M, N, K), B.make_mxfp4_desc(4, N, K)

    def step():
        a, _ = B.loka_mxfp4_linear(d, x, wq, sw)
        b, _ = B.loka_mxfp4_linear(d1, x[:4], w8, s8)
        q, s = B.loka_mxfp4_quantize(x, True)
        _, c = B.loka_mxfp4_gemm(B.make_mxfp4_desc(K, K, M), q, s, q, s, want_out=False, want_y=True)
        return a, b, c

    x.normal_(generator=_gen(0))
    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kept = step()
    for seed in (1, 2, 3):
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


def test_workspace_rules():
    M, K, N = 100, 512, 64
    d = B.make_mxfp4_desc(M, N, K)
    x, _, _ = _operand(M, K, 1)
    _, wq, sw = _operand(N, K, 2)
    need = B.lib().loka_mxfp4_linear_workspace(ctypes.byref(d))
    assert need >= M * K // 2 + M * K // 32
    with pytest.raises(B.LokaError) as e:
        B.loka_mxfp4_linear(d, x, wq, sw, workspace=torch.empty(need - 1, dtype=torch.uint8, device=DEV))
    assert e.value.status == B.LOKA_ERR_WORKSPACE
    want, _ = B.loka_mxfp4_linear(d, x, wq, sw)
    # what lies in the workspace does not matter, and nothing behind it is written
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device=DEV)
    got, _ = B.loka_mxfp4_linear(d, x, wq, sw, workspace=ws[:need])
    assert torch.equal(got, want) and bool((ws[need:] == 0xFF).all())
