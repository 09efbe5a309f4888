"""The workspace of attention over shared prefixes goes by the queries that a call can have, not by the rows of the tensor they lie in (no GPU
needed)."""
import ctypes
import os

import pytest

from paper_2604_18348_amd import binding as B
from tests.test_block_refusals import params


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    return B.load_library()


def size(lib, q_rows, groups, **kw):
    out = ctypes.c_size_t(7)
    assert lib.adacluster_prefix_workspace_bytes(ctypes.byref(params(q_rows=q_rows, **kw)), groups, ctypes.byref(out)) == 0
    return out.value


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("max_q", [1, 5])
@pytest.mark.parametrize("B_,groups,Hq,Hkv,d,pages", [(8, 1, 32, 8, 128, 2048), (64, 4, 32, 8, 128, 512), (3, 3, 8, 1, 64, 40), (300, 1, 4, 4, 64, 100)])
def test_spare_rows_cost_nothing(lib, B_, groups, Hq, Hkv, d, pages, max_q, dtype, bits):
    kw = dict(B=B_, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, bits=bits, max_pages=pages, max_q=max_q)
    need = size(lib, B_ * max_q, groups, **kw)
    for spare in (1, 100, 2048, 8192, 1 << 20):
        assert size(lib, B_ * max_q + spare, groups, **kw) <= need, spare
