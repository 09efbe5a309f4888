"""Attention over pages at soft-max scales above 1 / log2(e), where the lowest finite score times the scale is at the end of the range
of a float: rows that see nothing of a turn of keys, of a share of the list or at all, against the definition in 64 bits."""
import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within

pytestmark = pytest.mark.gpu

# at all of these, and at 0.97 and 1.53, -FLT_MAX / (scale log2(e)) times (scale log2(e)) rounds to minus infinity
SCALES = [0.88, 1.3, 2.72]


def _sees(p, sel, n, nq):
    """[nq, Hkv, n] from the lists [blocks, Hkv, topk] of one sequence (ascending, -1 behind the end), or of all pages."""
    see = torch.ones((nq, p.Hkv, n), dtype=torch.bool)
    if sel is not None:
        pages = -(-n // p.page)
        mark = torch.zeros((sel.shape[0], p.Hkv, pages + 1), dtype=torch.bool)
        mark.scatter_(2, torch.where(sel >= 0, sel, pages).long(), True)
        see = mark[..., :pages].repeat_interleave(p.page, 2)[..., :n].repeat_interleave(p.qblock, 0)[:nq].clone()
    if p.causal:
        see &= (torch.arange(n) <= n - nq + torch.arange(nq)[:, None])[:, None]
    return see


def _check(x, p, sel, o, lse):
    for b in range(x.B):
        k, v, ka, va = x.keys(b)
        n, nq = x.lens[b], x.news[b]
        see = _sees(p, None if sel is None else sel[b], n, nq)
        r = ref.attend(x.seq(x.q, b), k, v, see, p.softmax_scale, x.dtype, ka, va)
        at = slice(int(x.cu_q[b]), int(x.cu_q[b + 1]))
        _within(o[at], r["o"], r["o_tol"], "o of sequence %d" % b)
        _within(lse[at], r["lse"], r["lse_tol"], "lse of sequence %d" % b)


def _some_pages(x, p, seed):
    """Ascending lists of any pages of a sequence, its own or not: rows that see nothing of them are among those that do."""
    g = torch.Generator().manual_seed(seed)
    idx = torch.full((x.B, p.blocks, x.Hkv, p.topk), -1, dtype=torch.int32)
    for b in range(x.B):
        pages = -(-x.lens[b] // x.page)
        for i in range(p.blocks):
            for h in range(x.Hkv):
                n = min(pages, int(torch.randint(0, p.topk + 1, (1,), generator=g)))
                idx[b, i, h, :n] = torch.randperm(pages, generator=g)[:n].sort()[0].int()
    return idx


def _attend(layout, dtype, bits, scale, listed, causal):
    d, page, Hq, Hkv, lens, news, qblock, topk = layout
    x = Batch(dtype, bits, d, page, Hq, Hkv, lens, news, 41)
    p = x.params(qblock=qblock, topk=topk, causal=causal, softmax_scale=scale)
    p.softmax_scale = torch.tensor(scale, dtype=torch.float32).item()        # (as the call takes it)
    sel = _some_pages(x, p, 3) if listed else None
    o, lse = B.adacluster_block_attn(p, x.q.cuda(), x.cu_q.cuda(), cache=x.cache, sel_idx=None if sel is None else sel.cuda(), **x.where())
    _check(x, p, sel, o, lse)


FEW = [  # d, page, Hq, Hkv, lens, news, qblock, topk
    (64, 16, 4, 2, [100, 40, 9], [70, 40, 30], 16, 5),       # chunks; a sequence with more queries than keys
    (128, 64, 8, 2, [1100, 330, 40], [1, 1, 1], 1, 5),       # a last page whose second half holds no key; lists in shares
    (64, 16, 2, 1, [1000, 300], [40, 40], 20, 30),
]


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4), (F, 4)])
@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("layout", FEW)
def test_rows_that_see_nothing_of_a_turn(layout, scale, dtype, bits, listed, causal):
    _attend(layout, dtype, bits, scale, listed, causal)


MANY = [  # launches of the kernel for many rows
    (128, 16, 16, 4, [700, 333], [650, 400], 16, 9),
    (64, 32, 24, 8, [400, 97], [400, 120], 17, 7),
    (64, 16, 32, 16, [590, 301], [600, 600], 64, 20),
    (128, 64, 32, 16, [590, 301], [600, 600], 64, 4),
]


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("scale", [0.97, 1.53])
@pytest.mark.parametrize("layout,listed", [(MANY[0], True), (MANY[1], True), (MANY[2], True), (MANY[2], False), (MANY[3], False)])
def test_rows_that_see_nothing_of_a_tile(layout, listed, scale, causal):
    d, page, Hq, Hkv, lens, news, qblock, topk = layout
    G = Hq // Hkv
    qblock_run = qblock if listed else 128 // G
    assert qblock_run * G >= 33 and len(lens) * Hkv * -(-max(news) // qblock_run) >= 256
    _attend(layout, BF, 0, scale, listed, causal)


@pytest.mark.parametrize("dtype", [BF, F])
def test_gradients_at_a_scale_that_is_not_the_default(dtype):
    """Rows of weight zero among others, and rows that see nothing: their gradients are zero and reach no key."""
    for d, page, Hq, Hkv, qblock, topk in ((64, 16, 4, 2, 8, 3), (128, 64, 36, 1, 16, 2), (64, 64, 48, 1, 16, 2)):
        x = Batch(dtype, 0, d, page, Hq, Hkv, [150, 20], [150, 33], 30, paged=False)
        p = x.params(qblock=qblock, topk=topk)
        p.softmax_scale = torch.tensor(0.88, dtype=torch.float32).item()
        sel = _some_pages(x, p, 5)
        q, k, v, cu_q, cu_k = x.q.cuda(), x.k.cuda(), x.v.cuda(), x.cu_q.cuda(), x.cu_k.cuda()
        o, lse = B.adacluster_block_attn(p, q, cu_q, k=k, v=v, cu_k=cu_k, sel_idx=sel.cuda())
        _check(x, p, sel, o, lse)
        d_o = torch.randn(q.shape, generator=torch.Generator().manual_seed(2)).to(dtype)
        grads = B.adacluster_block_attn_backward(p, q, k, v, o, lse, d_o.cuda(), cu_q, cu_k, sel_idx=sel.cuda())
        for b in range(x.B):
            n, nq = x.lens[b], x.news[b]
            see = _sees(p, sel[b], n, nq)
            aq, ak = slice(int(x.cu_q[b]), int(x.cu_q[b + 1])), slice(int(x.cu_k[b]), int(x.cu_k[b + 1]))
            r = ref.attend(x.seq(x.q, b), x.seq(x.k, b), x.seq(x.v, b), see, p.softmax_scale, dtype, d_o=d_o[aq])
            for got, at, name in zip(grads, (aq, ak, ak), ("dq", "dk", "dv")):
                _within(got[at], r[name], r[name + "_tol"], "%s of sequence %d" % (name, b))
            none = ~see.any(-1)                              # [nq, Hkv]
            assert bool((grads[0][aq].view(nq, Hkv, -1, d).cpu()[none] == 0).all()) and bool(none.any())
