"""Attention over pages and autograd: the call alone records nothing and says so; inside a torch.autograd.Function it gives gradients."""
import math
import warnings

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within

pytestmark = pytest.mark.gpu


class PageAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, p, q, k, v, cu, sel):
        o, lse = B.adacluster_block_attn(p, q, cu, k=k, v=v, cu_k=cu, sel_idx=sel)
        ctx.p, ctx.cu, ctx.sel = p, cu, sel
        ctx.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, o, lse = ctx.saved_tensors
        d_o = d_o.contiguous()                               # (a sum's gradient is one number, broadcast: refused as it stands)
        return (None, *B.adacluster_block_attn_backward(ctx.p, q, k, v, o, lse, d_o, ctx.cu, ctx.cu, sel_idx=ctx.sel), None, None)


@pytest.mark.parametrize("name", ["q", "k", "v"])
def test_a_call_on_tensors_that_require_gradients_warns(name):
    x = Batch(BF, 0, 64, 16, 2, 1, [40], [40], 3, paged=False, spare=0)
    p, cu = x.params(), x.cu_q.cuda()
    t = dict(q=x.q.cuda(), k=x.k.cuda(), v=x.v.cuda())
    call = lambda: B.adacluster_block_attn(p, t["q"], cu, k=t["k"], v=t["v"], cu_k=cu)  # noqa: E731
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        want = call()
        t[name].requires_grad_()
        with torch.no_grad():
            call()
    with pytest.warns(UserWarning, match="records nothing for autograd"):
        got = call()
    assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, want))


def test_a_cache_does_not_warn_but_its_queries_do():
    x = Batch(BF, 0, 64, 16, 2, 1, [40], [1], 3)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        B.adacluster_block_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), cache=x.cache, **x.where())
    with pytest.warns(UserWarning, match="records nothing for autograd"):
        B.adacluster_block_attn(x.params(), x.q.cuda().requires_grad_(), x.cu_q.cuda(), cache=x.cache, **x.where())


@pytest.mark.parametrize("dtype", [BF, F])
def test_gradients_through_a_function(dtype):
    """Heads that share keys, two passes that add up, a tensor that enters twice; a gradient that is one number for all rows."""
    x = Batch(dtype, 0, 64, 16, 4, 2, [60, 33], [60, 33], 30, paged=False, spare=0)
    p, cu = x.params(qblock=8, topk=3), x.cu_q.cuda()
    q, k, v = (t.cuda().requires_grad_() for t in (x.q, x.k, x.v))
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        sel, _ = B.adacluster_block_select(p, q, cu, B.adacluster_block_boxes(p, k, cu), cu_k=cu)
        o = PageAttention.apply(p, q, k, v, cu, sel)
        d_o = torch.randn(o.shape, generator=torch.Generator().manual_seed(1)).to(dtype)
        o.backward(d_o.cuda())
    first = [t.grad.clone() for t in (q, k, v)]
    for b in range(2):
        n = x.lens[b]
        mark = torch.zeros((sel.shape[1], 2, -(-n // 16) + 1), dtype=torch.bool)
        mark.scatter_(2, torch.where(sel[b].cpu() >= 0, sel[b].cpu(), -(-n // 16)).long(), True)
        see = mark[..., :-1].repeat_interleave(16, 2)[..., :n].repeat_interleave(8, 0)[:n]
        see = see & (torch.arange(n) <= torch.arange(n)[:, None])[:, None]
        at = slice(int(x.cu_q[b]), int(x.cu_q[b + 1]))
        r = ref.attend(x.q[at], x.k[at], x.v[at], see, 1 / math.sqrt(64), dtype, d_o=d_o[at])
        for got, name in zip(first, ("dq", "dk", "dv")):
            _within(got[at], r[name], r[name + "_tol"], "%s of sequence %d" % (name, b))
    PageAttention.apply(p, q, k, v, cu, sel).backward(d_o.cuda())
    assert all(torch.equal(t.grad, 2 * g) for t, g in zip((q, k, v), first))
    PageAttention.apply(p, q, k, k, cu, sel).sum().backward()            # keys that are the values, a gradient of one number
    assert all(bool(t.grad.isfinite().all()) for t in (q, k))
