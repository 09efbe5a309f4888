"""Arguments that attention over shared prefixes, the weights of keys and eviction refuse, on the host and before anything is launched
(no GPU needed)."""
import ctypes
import os

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests.test_block_refusals import ONE, Z, message, params


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    return B.load_library()


def size(lib, c, groups=1):
    out = ctypes.c_size_t(7)
    return lib.adacluster_prefix_workspace_bytes(ctypes.byref(c), groups, ctypes.byref(out)), out.value


def prefix(lib, c, groups=1, ws=ONE, n=1 << 40, **kw):
    a = dict(q=ONE, cu_q=ONE, k=ONE, v=ONE, km=Z, vm=Z, lens=ONE, table=ONE, cu_group=ONE, prefix=ONE, o=ONE, lse=ONE)
    a.update(kw)
    return lib.adacluster_prefix_attn(ctypes.byref(c), groups, *a.values(), ws, n, Z)


def test_prefix(lib):
    assert size(lib, params())[0] == 0 and size(lib, params())[1] > 0 and size(lib, params())[1] % 256 == 0
    for c, groups, code in ((params(), -1, -2), (params(), 3, -2), (params(num_pages=0, k_rows=3), 1, -1), (params(d=96), 1, -2), (params(bits=3), 1, -3),
                            (params(Hq=65534, Hkv=1, q_rows=1 << 20, B=1), 1, -5)):
        assert size(lib, c, groups) == (code, 7) and message(lib)
        assert prefix(lib, c, groups) == code
    assert lib.adacluster_prefix_workspace_bytes(ctypes.byref(params()), 1, None) == -1
    assert lib.adacluster_prefix_workspace_bytes(None, 1, ctypes.byref(ctypes.c_size_t())) == -1
    for name in ("q", "cu_q", "k", "v", "lens", "table", "cu_group", "prefix", "o"):
        assert prefix(lib, params(), **{name: Z}) == -1, name
    for name in ("q", "k", "v", "o"):
        assert prefix(lib, params(), **{name: ctypes.c_void_p(264)}) == -1, name
    assert prefix(lib, params(bits=4)) == -1 and prefix(lib, params(bits=4), km=ONE) == -1
    for name in ("q_stride", "o_stride", "k_stride", "v_stride"):
        c = params()
        getattr(c, name)[1] = 12
        assert prefix(lib, c) == -1, name
    far = params()
    far.k_stride[1] = 1 << 25                                                     # tokens of a page far apart: another kernel, the same workspace
    assert size(lib, far) == size(lib, params())
    need = size(lib, params())[1]
    assert prefix(lib, params(), ws=Z) == -4 and prefix(lib, params(), ws=ctypes.c_void_p(272)) == -4 and prefix(lib, params(), n=need - 1) == -4


def weights(lib, c, decay=1.0, out=ONE, ws=ONE, n=1 << 40, **kw):
    a = dict(q=ONE, cu_q=ONE, lse=ONE, k=ONE, km=Z, lens=ONE, table=ONE, w=ONE)
    a.update(kw)
    return lib.adacluster_cache_weights(ctypes.byref(c), *a.values(), decay, out, ws, n, Z)


def test_weights(lib):
    for name in ("q", "cu_q", "lse", "k", "lens", "table", "out"):
        assert weights(lib, params(), **{name: Z}) == -1, name
    for name in ("q", "k", "w", "out"):
        assert weights(lib, params(), **{name: ctypes.c_void_p(264)}) == -1, name
    for decay in (-0.1, 1.5, float("nan"), float("inf")):
        assert weights(lib, params(), decay) == -1
    assert weights(lib, params(num_pages=0, k_rows=4)) == -1
    assert weights(lib, params(bits=4)) == -1
    assert weights(lib, params(d=32)) == -2
    c = params()
    c.k_stride[2] = 63
    assert weights(lib, c) == -1 and "16 bytes" in message(lib)
    out = ctypes.c_size_t(7)
    f = lib.adacluster_weights_workspace_bytes
    assert f(ctypes.byref(params(num_pages=0, k_rows=4)), ctypes.byref(out)) == -1 and f(ctypes.byref(params()), None) == -1 and f(None, ctypes.byref(out)) == -1
    assert f(ctypes.byref(params(B=1, Hkv=1, max_q=2000)), ctypes.byref(out)) == 0 and out.value > 0      # few keys for many rows: shares of them
    many = params(B=1, Hkv=1, max_q=2000)
    assert weights(lib, many, ws=Z) == -4 and weights(lib, many, n=out.value - 1) == -4 and weights(lib, many, ws=ctypes.c_void_p(272)) == -4
    assert weights(lib, params(B=1, Hq=65535, Hkv=1, max_q=1 << 20)) == -5


def evict(lib, c, keep=20, recent=2, **kw):
    a = dict(new_table=ONE, kept=ONE, new_lens=ONE, new_w=ctypes.c_void_p(512), k=ONE, v=ONE, km=Z, vm=Z, boxes=ONE)
    b = dict(lens=ONE, table=ONE, w=ONE)
    for d in (a, b):
        d.update({n: v for n, v in kw.items() if n in d})
    return lib.adacluster_cache_evict(ctypes.byref(c), *b.values(), keep, recent, *a.values(), Z)


def test_evict(lib):
    for name in ("lens", "table", "w", "new_table", "kept", "new_lens", "new_w", "k", "v", "boxes"):
        assert evict(lib, params(), **{name: Z}) == -1, name
    for keep, recent in ((0, 0), (-1, 0), ((1 << 29) + 1, 0), (20, -1), (20, 5), (15, 0)):      # (the first page is 16 tokens)
        assert evict(lib, params(keep_first=1), keep, recent) == -1, (keep, recent)
    assert "first pages" in message(lib)
    assert evict(lib, params(keep_first=1 << 30), 20, 2) == -1
    assert evict(lib, params(), new_w=ONE) == -1                                  # in place
    for name in ("w", "new_w"):
        assert evict(lib, params(), **{name: ctypes.c_void_p(264)}) == -1 and "16 bytes" in message(lib), name
    assert evict(lib, params(num_pages=0, k_rows=4)) == -1
    assert evict(lib, params(bits=4)) == -1
    c = params()
    c.v_stride[1] = 12
    assert evict(lib, c) == -1


def test_binding_checks_its_tensors():
    p = B.BlockParams(B=1, Hq=2, Hkv=1, d=64, page=16, max_pages=2, max_q=1)
    q, i = torch.zeros((1, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    cache = B.alloc_cache(p, 2, device="cpu")
    w = torch.zeros((1, 1, 32))
    with pytest.raises(ValueError, match="must be a"):                            # not on a GPU
        B.adacluster_prefix_attn(p, q, i, cache, i[:1], i.view(1, 2), i, i[:1])
    with pytest.raises(ValueError, match="must be a"):
        B.adacluster_cache_weights(p, q, i, w[0, 0, :2].view(1, 2), cache, i[:1], i.view(1, 2))
    with pytest.raises(ValueError, match="must be a"):
        B.adacluster_cache_evict(p, cache, i[:1], i.view(1, 2), w, 4, 1, i.view(1, 2))
    with pytest.raises(B.AdaClusterError):
        B.adacluster_prefix_workspace_bytes(p, 2, 1, 2)                           # more groups than sequences
    assert B.adacluster_prefix_workspace_bytes(p, 1, 0, 2) == 0
