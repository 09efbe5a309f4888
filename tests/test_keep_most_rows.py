"""The most rows a head of keys (queries times the heads that share it) that attention over shared prefixes and the weights of keys take: a tile of
rows past the last one still has numbers of 32 bits (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2604_18348_amd import binding as B
from tests.test_block_refusals import message, params
from tests.test_keep_overlap import PLACES as P, Z, at


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    return B.load_library()


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("less", [4, 16, 64, 128, 1020])
def test_refused(lib, less, dtype):
    n = 2 ** 29 - less // 4
    c = params(B=1, Hq=4, Hkv=1, max_q=n, q_rows=n, dtype=dtype)
    assert lib.adacluster_cache_weights(ctypes.byref(c), P["k"], P["lens"], P["boxes"], P["k"], Z, P["lens"], P["table"], P["w"], 0.5, P["new_w"],
                                        at(1 << 30), 1 << 40, Z) == -5 and "2^31 - 1024" in message(lib)
    assert lib.adacluster_prefix_workspace_bytes(ctypes.byref(c), 1, ctypes.byref(ctypes.c_size_t())) == -5 and "2^31 - 1024" in message(lib)


def test_taken(lib):
    c, out = params(B=1, Hq=4, Hkv=1, max_q=2 ** 29 - 256, q_rows=2 ** 29 - 256), ctypes.c_size_t()
    assert lib.adacluster_prefix_workspace_bytes(ctypes.byref(c), 1, ctypes.byref(out)) == 0 and out.value
