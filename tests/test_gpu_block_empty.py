"""Attention over pages where a call has no queries, no keys or neither: outputs and gradients are those of rows that see nothing."""
import math

import pytest
import torch

from paper_2604_18348_amd import binding as B

pytestmark = pytest.mark.gpu

KINDS = [(torch.bfloat16, 64), (torch.float32, 128)]


def _params(dtype, d, **kw):
    return B.BlockParams(B=2, Hq=4, Hkv=2, d=d, dtype=B.BF16 if dtype == torch.bfloat16 else B.F32, page=16, max_pages=3, topk=3, **kw)


def _cu(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rand(rows, heads, d, dtype):
    return torch.randn((rows, heads, d), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("listed", [False, True])
def test_queries_without_keys(dtype, d, listed):
    """Rows of a sequence: output 0, lse -inf, gradient 0.  The row behind the last sequence stays as it was."""
    p = _params(dtype, d, max_q=3, qblock=2)
    q, d_o, k = _rand(6, 4, d, dtype), _rand(6, 4, d, dtype), _rand(0, 2, d, dtype)
    cu_q, cu_k = _cu(0, 3, 5), _cu(0, 0, 0)
    sel = None
    if listed:
        boxes = B.adacluster_block_boxes(p, k, cu_k)
        assert boxes.shape == (2, 3, 2, 2, d) and not bool(boxes.any())
        for rows in (None, 0):
            sel, cnt = B.adacluster_block_select(p, q, cu_q, boxes, cu_k=cu_k, k_rows=rows)
            assert bool((sel == -1).all()) and not bool(cnt.any())
    for cu in (cu_k, _cu(0, 7, 9)):                          # (prefixes past the rows are held to them)
        out, lse = torch.full_like(q, 7.0), torch.full((6, 4), 7.0, device="cuda")
        o, l = B.adacluster_block_attn(p, q, cu_q, k=k, v=k, cu_k=cu, sel_idx=sel, out=out, lse=lse)
        assert bool((o[:5] == 0).all()) and bool((l[:5] == -math.inf).all()) and bool((o[5] == 7).all()) and bool((l[5] == 7).all())
        outs = [torch.full_like(t, 7.0) for t in (q, k, k)]
        dq, dk, dv = B.adacluster_block_attn_backward(p, q, k, k, o, l, d_o, cu_q, cu, sel_idx=sel, outs=outs)
        assert bool((dq[:5] == 0).all()) and bool((dq[5] == 7).all()) and dk.shape == dv.shape == (0, 2, d)
        dq, dk, dv = B.adacluster_block_attn_backward(p, q, k, k, o, l, d_o, cu_q, cu, sel_idx=sel)
        assert bool((dq == 0).all()) and dk.shape == dv.shape == (0, 2, d)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("max_q", [1, 0])
@pytest.mark.parametrize("listed", [False, True])
def test_gradients_of_a_step_without_queries(dtype, d, max_q, listed):
    """Every key of a sequence has gradient 0; the rows behind the last sequence stay as they were."""
    p = _params(dtype, d, max_q=max_q)
    q, k, v = _rand(0, 4, d, dtype), _rand(50, 2, d, dtype), _rand(50, 2, d, dtype)
    cu_q, cu_k = _cu(0, 0, 0), _cu(0, 40, 47)
    sel = None
    if listed:
        sel, cnt = B.adacluster_block_select(p, q, cu_q, B.adacluster_block_boxes(_params(dtype, d), k, cu_k), cu_k=cu_k)
    o, lse = B.adacluster_block_attn(p, q, cu_q, k=k, v=v, cu_k=cu_k, sel_idx=sel)
    assert o.shape == (0, 4, d) and lse.shape == (0, 4)
    outs = [torch.full_like(t, 7.0) for t in (q, k, v)]
    dq, dk, dv = B.adacluster_block_attn_backward(p, q, k, v, o, lse, o, cu_q, cu_k, sel_idx=sel, outs=outs)
    assert dq.shape == (0, 4, d)
    for t in (dk, dv):
        assert bool((t[:47] == 0).all()) and bool((t[47:] == 7).all())
    dq, dk, dv = B.adacluster_block_attn_backward(p, q, k, v, o, lse, o, cu_q, cu_k, sel_idx=sel)
    assert dq.shape == (0, 4, d) and not bool(dk.any()) and not bool(dv.any())


@pytest.mark.parametrize("dtype,d", KINDS)
def test_neither_queries_nor_keys(dtype, d):
    p = _params(dtype, d)
    q, k, cu = _rand(0, 4, d, dtype), _rand(0, 2, d, dtype), _cu(0, 0, 0)
    assert not bool(B.adacluster_block_boxes(p, k, cu).any())
    o, lse = B.adacluster_block_attn(p, q, cu, k=k, v=k, cu_k=cu)
    grads = B.adacluster_block_attn_backward(p, q, k, k, o, lse, o, cu, cu)
    assert [tuple(t.shape) for t in grads] == [(0, 4, d), (0, 2, d), (0, 2, d)]
    with pytest.raises(ValueError):                          # arguments are looked at all the same
        B.adacluster_block_attn_backward(p, q, k, k, o, lse, o, cu, cu[:2])
