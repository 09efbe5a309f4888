"""Arguments that the calls of attention over pages refuse, on the host and before anything is launched (no GPU needed)."""
import ctypes
import os
import re
import struct

import pytest

from paper_2604_18348_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
Z, ONE = ctypes.c_void_p(0), ctypes.c_void_p(256)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    return B.load_library()


def params(num_pages=8, q_rows=4, k_rows=0, strides=True, **kw):
    base = dict(B=2, Hq=4, Hkv=2, d=64, page=16, max_pages=8, max_q=2, topk=4)
    base.update(kw)
    c = B.CBlockParams.from_buffer_copy(B._block_c(B.BlockParams(**base), q_rows, k_rows, num_pages))
    if strides:
        for name, n in B.CBlockParams._fields_[17:]:
            for i in range(n._length_):
                getattr(c, name)[i] = 64
    return c


def message(lib):
    buf = ctypes.create_string_buffer(256)
    lib.adacluster_last_error(buf, 256)
    return buf.value.decode()


def size(lib, c, call=B.BLOCK_ATTN):
    out = ctypes.c_size_t(7)
    return lib.adacluster_block_workspace_bytes(ctypes.byref(c), call, ctypes.byref(out)), out.value


def test_struct_matches_the_header():
    src = open(os.path.join(ROOT, "include", "adacluster.h")).read()
    body = src[src.index("typedef struct adacluster_block_params {"):src.index("} adacluster_block_params;")]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip() for f in re.findall(r"\b(?:int32_t|int64_t|float)\s+([^;]+);", body) for n in f.split(",")]
    mine = [n if not hasattr(t, "_length_") else "%s[%d]" % (n, t._length_) for n, t in B.CBlockParams._fields_]
    assert names == mine
    assert struct.calcsize("@16if22q") == ctypes.sizeof(B.CBlockParams)
    c = B.CBlockParams.from_buffer_copy(B._block_c(B.BlockParams(B=3, Hq=8, Hkv=4, d=64, topk=9, softmax_scale=0.5), 5, 6, 7, q=(1, 2), dv=(3, 4)))
    assert (c.B, c.Hq, c.num_pages, c.topk, c.q_rows, c.k_rows, c.softmax_scale) == (3, 8, 7, 9, 5, 6, 0.5)
    assert list(c.q_stride) == [1, 2] and list(c.dv_stride) == [3, 4] and list(c.dk_stride) == [0, 0]


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -2), (dict(B=65536), -2), (dict(Hq=5), -2), (dict(Hkv=0), -2), (dict(d=96), -2), (dict(d=256), -2), (dict(dtype=2), -3),
    (dict(bits=8), -3), (dict(page=8), -2), (dict(page=48), -2), (dict(page=256), -2), (dict(max_pages=0), -2), (dict(max_pages=1 << 27), -2),
    (dict(max_q=0), -2), (dict(qblock=0), -2), (dict(qblock=1025), -2), (dict(causal=2), -1), (dict(topk=-1), -1), (dict(keep_first=-1), -1),
    (dict(q_rows=0), -2), (dict(k_rows=-1), -2), (dict(num_pages=-1), -2), (dict(softmax_scale=float("nan")), -1),
    (dict(softmax_scale=float("inf")), -1), (dict(softmax_scale=1e31), -1), (dict(B=60000, max_q=1 << 29), -2),
    (dict(max_q=(1 << 29) + 1), -2), (dict(max_pages=(1 << 25) + 1), -2),
])
def test_parameters(lib, kw, code):
    assert size(lib, params())[0] == 0
    rc, n = size(lib, params(**kw))
    assert rc == code and n == 7 and message(lib)


def test_workspace_sizes(lib):
    assert size(lib, params(), 3)[0] == -1
    assert lib.adacluster_block_workspace_bytes(None, 0, ctypes.byref(ctypes.c_size_t())) == -1
    assert lib.adacluster_block_workspace_bytes(ctypes.byref(params()), 0, None) == -1
    big = params(B=1, max_pages=8192, max_q=1)                                     # few records, many pages: scores in memory
    assert size(lib, big, B.BLOCK_SELECT)[1] >= 2 * 8192 * 8


def append(lib, c, **kw):
    a = dict(k=ONE, v=ONE, cu=ONE, lens=ONE, table=ONE, kp=ONE, vp=ONE, km=Z, vm=Z, boxes=ONE)
    a.update(kw)
    return lib.adacluster_cache_append(ctypes.byref(c), *a.values(), Z)


def read(lib, c, **kw):
    a = dict(cu=ONE, first=ONE, table=ONE, kp=ONE, vp=ONE, km=Z, vm=Z, k=ONE, v=ONE)
    a.update(kw)
    return lib.adacluster_cache_read(ctypes.byref(c), *a.values(), Z)


def test_cache_calls(lib):
    for call, need in ((append, ("k", "v", "cu", "lens", "table", "kp", "vp", "boxes")), (read, ("cu", "first", "table", "kp", "vp", "k", "v"))):
        for name in need:
            assert call(lib, params(), **{name: Z}) == -1, name
        assert call(lib, params(num_pages=0)) == -1
        assert call(lib, params(bits=4)) == -1                                   # no (step, lowest) pairs
        assert call(lib, params(bits=4), km=ONE, vm=ctypes.c_void_p(260)) == -1   # misaligned
        assert call(lib, params(), k=ctypes.c_void_p(264)) == -1
        odd = params()
        odd.k_stride[1] = 63
        assert call(lib, odd) == -1 and "16 bytes" in message(lib)
        neg = params()
        neg.v_stride[0] = -64
        assert call(lib, neg) == -1
    odd = params()
    odd.new_v_stride[0] = 4
    assert append(lib, odd) == -1
    assert lib.adacluster_cache_append(None, *[ONE] * 10, Z) == -1


def test_boxes(lib):
    f = lib.adacluster_block_boxes
    c = params(num_pages=0, k_rows=9)
    assert f(ctypes.byref(params()), ONE, ONE, ONE, Z) == -1                      # a pool keeps its own
    for args in ((Z, ONE, ONE), (ONE, Z, ONE), (ONE, ONE, Z)):
        assert f(ctypes.byref(c), *args, Z) == -1
    assert f(ctypes.byref(params(num_pages=0, k_rows=0)), ONE, ONE, ONE, Z) == -2


def select(lib, c, ws=ONE, n=1 << 30, **kw):
    a = dict(q=ONE, cu_q=ONE, cu_k=Z, lens=ONE, table=ONE, boxes=ONE, idx=ONE, cnt=ONE)
    a.update(kw)
    return lib.adacluster_block_select(ctypes.byref(c), *a.values(), ws, n, Z)


def test_select(lib):
    for name in ("q", "cu_q", "lens", "table", "boxes", "idx", "cnt"):
        assert select(lib, params(), **{name: Z}) == -1, name
    assert select(lib, params(num_pages=0, k_rows=5)) == -1                      # packed keys without cu_k
    assert select(lib, params(topk=0)) == -1
    # own pages of a block: ceil((qblock - 1) / page) + 1
    assert select(lib, params(topk=1)) == -1                                      # and the first page
    assert select(lib, params(topk=3, qblock=34, keep_first=0)) == -1
    assert "own positions" in message(lib)
    assert select(lib, params(topk=1, causal=0, keep_first=2)) == -1
    assert select(lib, params(), boxes=ctypes.c_void_p(258)) == -1
    big = params(B=1, max_pages=8192, max_q=1)
    assert select(lib, big, ws=Z) == -4
    assert select(lib, big, ws=ctypes.c_void_p(272)) == -4
    assert select(lib, big, n=8) == -4 and "too small" in message(lib)


def attn(lib, c, ws=ONE, n=1 << 30, **kw):
    a = dict(q=ONE, cu_q=ONE, k=ONE, v=ONE, km=Z, vm=Z, cu_k=Z, lens=ONE, table=ONE, sel=Z, o=ONE, lse=ONE)
    a.update(kw)
    return lib.adacluster_block_attn(ctypes.byref(c), *a.values(), ws, n, Z)


def test_attention(lib):
    for name in ("q", "cu_q", "k", "v", "lens", "table", "o"):
        assert attn(lib, params(), **{name: Z}) == -1, name
    assert attn(lib, params(num_pages=0, k_rows=5)) == -1
    assert attn(lib, params(num_pages=0, k_rows=0), cu_k=ONE) == -2
    assert attn(lib, params(num_pages=0, k_rows=5, bits=4), cu_k=ONE, km=ONE, vm=ONE) == -5
    assert attn(lib, params(topk=0), sel=ONE) == -1
    for name in ("q_stride", "o_stride", "k_stride", "v_stride"):
        c = params()
        getattr(c, name)[1] = 12
        assert attn(lib, c) == -1, name
    long = params(B=1, Hq=1, Hkv=1, max_pages=4096, max_q=1)
    assert size(lib, long)[1] > 0                                                 # its list is split: partial results
    assert attn(lib, long, ws=Z) == -4 and attn(lib, long, n=16) == -4


def backward(lib, c, ws=ONE, n=1 << 30, **kw):
    a = dict(q=ONE, k=ONE, v=ONE, o=ONE, lse=ONE, d_o=ONE, cu_q=ONE, cu_k=ONE, sel=Z, dq=ONE, dk=ONE, dv=ONE)
    a.update(kw)
    return lib.adacluster_block_attn_backward(ctypes.byref(c), *a.values(), ws, n, Z)


def test_backward(lib):
    good = lambda **kw: params(num_pages=0, k_rows=9, **kw)  # noqa: E731
    for name in ("q", "k", "v", "o", "lse", "d_o", "cu_q", "cu_k", "dq", "dk", "dv"):
        assert backward(lib, good(), **{name: Z}) == -1, name
    assert backward(lib, params(k_rows=9)) == -5                                  # gradients of a paged cache
    assert backward(lib, good(bits=4)) == -5
    assert backward(lib, good(topk=0), sel=ONE) == -1
    for name in ("q_stride", "o_stride", "do_stride", "dq_stride", "dk_stride", "dv_stride"):
        c = good()
        getattr(c, name)[0] = 2
        assert backward(lib, c) == -1, name
    assert backward(lib, good(), ws=Z) == -4 and backward(lib, good(), n=4) == -4


def test_binding_checks_its_tensors():
    import torch
    p = B.BlockParams(B=1, Hq=2, Hkv=1, d=64, page=16, max_pages=2, max_q=1, topk=2)
    q, cu = torch.zeros((1, 2, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be a"):                            # not on a GPU
        B.adacluster_block_attn(p, q, cu, k=q, v=q, cu_k=cu)
    with pytest.raises(ValueError, match="must be a"):
        B.adacluster_block_boxes(p, q[:, :1], cu)
    with pytest.raises(B.AdaClusterError):
        B.adacluster_block_workspace_bytes(B.BlockParams(B=1, Hq=3, Hkv=2, d=64), B.BLOCK_ATTN, 1)
