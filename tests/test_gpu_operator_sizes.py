"""Sizes whose work is more than one launch holds (2^32 threads): MXFP4 quantization and products, and the residual norm, in several
launches."""
import pytest
import torch

import plain_ops as P
from paper_2605_10886_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _e2m1(codes):
    v = torch.tensor(P.E2M1, device=DEV)
    return torch.cat((v, -v))[codes.int()]


def test_quantizing_down_the_longest_column():
    rows = (1 << 31) - 1               # 2^23 workgroups of 512 threads
    x = torch.zeros(rows, 1, dtype=torch.bfloat16, device=DEV)
    first, last = slice(0, 640), slice((rows - 640) // 32 * 32, rows)
    for part in (first, last):
        x[part] = torch.randn(x[part].shape, device=DEV, generator=_gen(part.start)).bfloat16()
    q, s = B.loka_mxfp4_quantize(x, True)
    assert q.shape == (1, 1 << 30) and s.shape == (1, 1 << 26)
    for part in (first, last):
        wq, ws = P.mx_quantize(x[part].t())
        n = -(-(part.stop - part.start) // 32)
        at = part.start // 32
        assert torch.equal(q[:, at * 16: (at + n) * 16], wq[:, :n * 16]) and torch.equal(s[:, at: at + n], ws[:, :n])
    assert not bool(q[:, first.stop // 2: last.start // 2].any()) and not bool(s[:, first.stop // 32: last.start // 32].any())


def test_quantizing_the_most_rows():
    rows = (1 << 30) + 261             # 2^24 + 5 workgroups of 256 threads; stored form 64 GiB
    x = torch.zeros(rows, 1, dtype=torch.bfloat16, device=DEV)
    for part in (slice(0, 1000), slice(rows - 1000, rows)):         # (one value a group: 1.5 times a power of two is exact)
        x[part] = (1.5 * torch.exp2(torch.randint(-9, 9, (1000, 1), device=DEV, generator=_gen(part.start)).float())).bfloat16()
    q, s = B.loka_mxfp4_quantize(x)
    assert torch.equal(B.loka_mxfp4_dequantize(q, s, 1), x)
    assert torch.equal(q[-1000:], P.mx_quantize(x[-1000:])[0]) and torch.equal(s[-1000:], P.mx_quantize(x[-1000:])[1])


def test_a_token_through_the_most_columns():
    N = (1 << 28) + 37                 # 2^23 + 2 workgroups of 512 threads
    codes = torch.randint(0, 16, (N,), dtype=torch.uint8, device=DEV, generator=_gen(1))
    wq = torch.zeros(N, 64, dtype=torch.uint8, device=DEV)
    wq[:, 0] = codes
    sw = torch.full((N, 4), 127, dtype=torch.uint8, device=DEV)
    out, _ = B.loka_mxfp4_linear(B.make_mxfp4_desc(1, N, 1), torch.ones(1, 1, dtype=torch.bfloat16, device=DEV), wq, sw)
    assert torch.equal(out[0], _e2m1(codes).bfloat16())


def test_the_most_problems():
    G = (1 << 23) + 5                  # a workgroup of 512 threads each
    codes = torch.randint(0, 16, (G,), dtype=torch.uint8, device=DEV, generator=_gen(2))
    xq = torch.zeros(G, 64, dtype=torch.uint8, device=DEV)
    xq[:, 0] = codes
    sx = torch.full((G, 4), 127, dtype=torch.uint8, device=DEV)
    wq, sw = B.loka_mxfp4_quantize(torch.ones(1, 1, dtype=torch.bfloat16, device=DEV))
    out, y = B.loka_mxfp4_gemm(B.make_mxfp4_desc(1, 1, 1, G, shared_w=True), xq, sx, wq, sw, want_y=True)
    assert torch.equal(y.view(-1), _e2m1(codes)) and torch.equal(out.view(-1), _e2m1(codes).bfloat16())


def test_the_norm_of_the_most_rows():
    rows, cols = (1 << 28) + 23, 16    # 2^24 + 2 workgroups of 256 threads
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    head, tail = (torch.randn(n, cols, device=DEV, generator=_gen(n)).bfloat16() for n in (50, 60))
    x[:50], x[-60:] = head, tail
    got = B.loka_add_rmsnorm(x, None, None, 1e-5, out=B.RMS_OUT_BF16)
    for part, alone in ((slice(0, 50), head), (slice(rows - 60, rows), tail)):
        assert torch.equal(got.y[part], B.loka_add_rmsnorm(alone, None, None, 1e-5, out=B.RMS_OUT_BF16).y)
    assert not bool(got.y[50:-60].view(torch.int32).any())
