"""Limits of the MXFP4 entry points' sizes, on the host."""
import ctypes

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
