"""Which kernel form the library chooses for the products that the GPU tests run, so that a changed choice cannot leave a form untested."""
import ctypes

import pytest

import mxfp4_shapes as S
from paper_2605_10886_amd import binding as B


@pytest.mark.parametrize("form,M,N,K,batch", S.ALL)
def test_the_tested_products_reach_their_forms(form, M, N, K, batch):
    d = B.make_mxfp4_desc(M, N, K, batch)
    L = B.lib()
    room = L.loka_mxfp4_gemm_workspace(ctypes.byref(d))
    assert L.loka_test_mxfp4_form(ctypes.byref(d)) == (S.HALVES if form == S.SPLIT else form)
    splits, rest = divmod(room, M * N * batch * 4)
    assert rest == 0 and (splits >= 2 if form == S.SPLIT else splits == 0)


def test_the_query_refuses_what_the_call_refuses():
    d = B.make_mxfp4_desc(0, 8, 8)
    assert B.lib().loka_test_mxfp4_form(ctypes.byref(d)) == -1 == B.lib().loka_test_mxfp4_form(None)
