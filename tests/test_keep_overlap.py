"""Outputs of eviction and of the weights of keys that lie over their inputs: refused on the host where workgroups would read what others
write (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2604_18348_amd import binding as B
from tests.test_block_refusals import Z, message, params


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    return B.load_library()


def at(n):
    return ctypes.c_void_p(n)


# places far apart, 2^24 bytes each
PLACES = {n: at((i + 1) << 24) for i, n in enumerate(("lens", "table", "w", "new_table", "kept", "new_lens", "new_w", "k", "v", "boxes"))}


def evict(lib, c, keep=20, recent=2, **kw):
    a = {**PLACES, **kw}
    return lib.adacluster_cache_evict(ctypes.byref(c), a["lens"], a["table"], a["w"], keep, recent, a["new_table"], a["kept"], a["new_lens"], a["new_w"],
                                      a["k"], a["v"], Z, Z, a["boxes"], Z)


def test_new_lens_in_place_of_seq_lens(lib):
    c = params(B=4)
    here = PLACES["lens"].value
    for to in (here, here + 4, here + 12, here - 4, here - 12):      # (four lengths each)
        assert evict(lib, c, new_lens=at(to)) == -1 and "new_lens" in message(lib), to - here


def test_new_weights_over_part_of_weights(lib):
    c = params(B=2, Hkv=2, max_pages=8)                          # 2 x 2 x 8 x 16 weights: 2048 bytes
    here = PLACES["w"].value
    for off in (0, 16, 512, 2032, -16, -2032):
        assert evict(lib, c, new_w=at(here + off)) == -1 and "new_weights" in message(lib), off
        if off:                                                  # (the weights of keys may be added to in place)
            assert lib.adacluster_cache_weights(ctypes.byref(c), PLACES["k"], PLACES["lens"], PLACES["boxes"], PLACES["k"], Z, PLACES["lens"], PLACES["table"],
                                                PLACES["w"], 0.5, at(here + off), Z, 0, Z) == -1 and "new_weights" in message(lib), off
