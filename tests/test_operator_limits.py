"""Limits of the MXFP4 entry points' sizes, on the host."""
import ctypes

import pytest
import torch

from paper_2605_10886_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)
MOST = (1 << 31) - 1


def test_more_than_any_memory_holds_is_refused():
    L = B.lib()
    for tr in (0, 1):
        assert L.loka_mxfp4_quantize(FAKE, MOST, 1 << 18, 1 << 18, tr, FAKE, FAKE, None) == B.LOKA_ERR_SHAPE
    assert L.loka_mxfp4_dequantize(FAKE, FAKE, MOST, MOST, FAKE, MOST, None) == B.LOKA_ERR_SHAPE
    for M, N, K, batch in ((MOST, 1, MOST, 1), (1, MOST, MOST, 1), (MOST, MOST, 1, 1), (1 << 16, 1 << 16, 1, MOST)):
        d = B.make_mxfp4_desc(M, N, K, batch)
        assert L.loka_mxfp4_gemm(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, None, 0, None) == B.LOKA_ERR_SHAPE, (M, N, K, batch)
        assert L.loka_mxfp4_gemm_workspace(ctypes.byref(d)) == 0


def test_the_layer_reads_no_strides():
    x, q, s = torch.zeros(8, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8)
    for name in ("strideX", "strideW", "strideO"):
        for v in (-128, 5, 1 << 62):
            d = B.make_mxfp4_desc(8, 8, 64)
            setattr(d, name, v)
            with pytest.raises(AssertionError, match="one GPU"):      # (past the descriptor: what is left is that the tensors are here)
                B.loka_mxfp4_linear(d, x, q, s)
    with pytest.raises(B.LokaError):
        B.loka_mxfp4_linear(B.make_mxfp4_desc(8, 8, 0), x, q, s)


def test_one_problem_reads_no_strides():
    q, s = torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(8, 4, dtype=torch.uint8)
    for name in ("strideX", "strideW", "strideO"):
        d = B.make_mxfp4_desc(8, 8, 64)
        setattr(d, name, -128)
        with pytest.raises(AssertionError, match="one GPU"):
            B.loka_mxfp4_gemm(d, q, s, q, s)
        d = B.make_mxfp4_desc(8, 8, 64, 2)
        setattr(d, name, -128)
        with pytest.raises(B.LokaError) as e:
            B.loka_mxfp4_gemm(d, q, s, q, s)
        assert e.value.status == B.LOKA_ERR_SHAPE


def test_a_workspace_is_one_run_of_memory():
    # bytes of an expanded or strided tensor are not its own: writing them would run past it or between its elements
    x, q, s = torch.zeros(64, 64, dtype=torch.bfloat16), torch.zeros(64, 64, dtype=torch.uint8), torch.zeros(64, 4, dtype=torch.uint8)
    hq, hs, rstd = torch.zeros(64, 64, dtype=torch.uint8), torch.zeros(64), torch.zeros(64)
    d = B.make_mxfp4_desc(64, 64, 64)
    for ws in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2]):
        for call in (lambda: B.loka_mxfp4_gemm(d, q, s, q, s, workspace=ws), lambda: B.loka_mxfp4_linear(d, x, q, s, workspace=ws),
                     lambda: B.loka_rmsnorm_backward(x, hq, hs, rstd, ckpt_mode=B.SCALE_ROW, workspace=ws)):
            with pytest.raises(AssertionError, match="workspace"):
                call()
