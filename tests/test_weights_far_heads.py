"""Which query strides the kernel of cache_weights for many rows takes: it holds an offset inside a stage of 64 rows in 32 bits, and heads that share
a key may be many and far apart.  Over 4 bits that kernel has a workspace and the one for few rows none, so the host's size tells which runs (no GPU
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


def farthest(G, d, token, head):
    """Bytes from a stage's first token to behind the farthest piece of its 64 rows, by going through them from every first head."""
    far = 0
    for first in {0, G - 1, max(0, G - 63), max(0, G - 64)}:
        for row in range(first, first + 64):
            far = max(far, row // G * token + row % G * head)
        far = max(far, (G - 1) * head)
    return 2 * (far + d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 64, 65, 96, 129, 130, 160, 256, 1000, 4096])
def test_offsets_of_a_stage_fit_32_bits(lib, G, d):
    c = params(B=1, Hq=G, Hkv=1, d=d, bits=4, max_q=64, q_rows=64)
    taken = 0
    near = [(2 ** 31 - 64) // G // 8 * 8 + 8 * i for i in (-40, -1, 0, 1, 40)]
    for head in sorted({64, 1 << 14, 1 << 20, (1 << 23) - 64, 1 << 23, (1 << 24) - 64, 1 << 24, 1 << 31, 1 << 32, 1 << 40, 1 << 60, *near}):
        for token in (64, G * d, 1 << 20, (1 << 24) - 64, 1 << 24, 1 << 25, 1 << 31, 1 << 32, 1 << 60):
            c.q_stride[0], c.q_stride[1] = token, head
            out = ctypes.c_size_t(7)
            assert lib.adacluster_weights_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == 0
            if out.value:
                assert farthest(G, d, token, head) <= 2 ** 32, (token, head)
                taken += 1
    assert taken                                                 # strides of ordinary tensors among them
    c.q_stride[0], c.q_stride[1] = G * d, d
    assert lib.adacluster_weights_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == 0 and out.value
