"""Attention of up to 16 rows a block over 16-bit keys: the weights lose nothing in the product with the values, so that the output is
off by its own rounding to bfloat16 and by what products in 32 bits and weights of 16 bits of fraction leave.  Scores in fp32."""
import math

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,page,Hq,Hkv,lens,news,qblock,paged", [
    (64, 16, 8, 1, [40, 7, 1], [1, 1, 1], 1, True),          # few keys: no error averages out
    (128, 64, 8, 2, [1000, 300], [1, 1], 1, True),
    (128, 16, 3, 1, [5000], [5], 5, True),                   # a list in shares
    (64, 32, 4, 4, [77, 16], [77, 16], 4, False),
])
@pytest.mark.parametrize("spread", [1.0, 6.0])
def test_outputs_are_off_by_their_own_rounding(d, page, Hq, Hkv, lens, news, qblock, paged, spread):
    x = Batch(BF, 0, d, page, Hq, Hkv, lens, news, 61, paged=paged)
    p = x.params(qblock=qblock, topk=max(1, x.max_pages), keep_first=0, softmax_scale=spread / math.sqrt(d))
    p.softmax_scale = torch.tensor(p.softmax_scale, dtype=torch.float32).item()
    idx = torch.arange(p.topk, dtype=torch.int32, device="cuda").expand(x.B, p.blocks, Hkv, p.topk).contiguous()      # (lists: blocks stay small)
    keys = dict(cache=x.cache) if paged else dict(k=x.k.cuda(), v=x.v.cuda())
    o, lse = B.adacluster_block_attn(p, x.q.cuda(), x.cu_q.cuda(), sel_idx=idx, **keys, **x.where())
    for b in range(x.B):
        n, nq = x.lens[b], x.news[b]
        see = ref.sees(None, n, nq, Hkv, page, qblock, 1)
        q, k, v = x.seq(x.q, b), x.seq(x.k, b), x.seq(x.v, b)
        r = ref.attend(q, k, v, see, p.softmax_scale, F)     # (bounds without a rounding of the weights)
        weighed = ref.attend(q, k, v.abs(), see, p.softmax_scale, F)["o"]
        at = slice(int(x.cu_q[b]), int(x.cu_q[b + 1]))
        _within(o[at], r["o"], r["o_tol"] + 1.01 * (2.0 ** -16 * weighed + ref.half(BF) * r["o"].abs()), "o of sequence %d" % b)
        _within(lse[at], r["lse"], r["lse_tol"], "lse of sequence %d" % b)


@pytest.mark.parametrize("Hq,nq", [(1, 1), (4, 30)])
def test_scores_in_fp32_are_two_sums(Hq, nq):
    """One key, so lse is the score: 1 and 127 terms of 1.5 2^-27, each of them (and four together) below half a step of 1.  One chain of sums
    leaves 1; of two chains one keeps its 64 terms, 96 * 2^-27 = 7.2e-7.  The logarithm's two roundings take 2.4e-7 of it at most."""
    d = 128
    p = B.BlockParams(B=1, Hq=Hq, Hkv=1, d=d, dtype=B.F32, page=16, max_pages=1, max_q=nq, causal=0, softmax_scale=1.0)
    q = torch.ones((nq, Hq, d), device="cuda")
    cu_q, cu_k = (torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (nq, 1))
    got = []
    for rest in (0.0, 1.5 * 2.0 ** -27):
        k = torch.full((1, 1, d), rest, device="cuda")
        k[..., 0] = 1
        got.append(B.adacluster_block_attn(p, q, cu_q, k=k, v=k, cu_k=cu_k)[1].double())
    assert bool(((got[0] - 1).abs() <= 2.0 ** -22).all())
    assert bool((got[1] - got[0] >= 96 * 2.0 ** -27 - 2.4e-7).all()), (got[1] - got[0]).min()
