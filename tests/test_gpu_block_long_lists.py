"""Attention over pages where a workgroup looks up its list of pages in several goes (512 pages at a time), and where the rows of a block
belong to several workgroups of the kernels for many rows; the launch that is meant is worked out beside each case."""
import math

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within

pytestmark = pytest.mark.gpu

HELD = 512                                                   # pages looked up at a time


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


def _check(x, p, sel, o, lse, rows=None):
    """rows: at most so many queries of a sequence, the first, the last and others between them."""
    for b in range(x.B):
        n, nq = x.lens[b], x.news[b]
        k, v, ka, va = x.keys(b)
        at = torch.arange(nq)
        if rows and rows < nq:
            at = torch.linspace(0, nq - 1, rows).round().long()
        see = _sees(p, None if sel is None else sel[b].cpu(), n, nq)[at]
        r = ref.attend(x.seq(x.q, b)[at], k, v, see, 1 / math.sqrt(x.d), x.dtype, ka, va)
        to = (int(x.cu_q[b]) + at).to(o.device)
        _within(o[to], r["o"], r["o_tol"], "o of sequence %d" % b)
        _within(lse[to], r["lse"], r["lse_tol"], "lse of sequence %d" % b)


def _long_lists(x, p, pages_of, seed):
    """Ascending lists of pages_of(pages) pages that are spread over the whole sequence, the last page among them."""
    g = torch.Generator().manual_seed(seed)
    idx = torch.full((x.B, p.blocks, x.Hkv, p.topk), -1, dtype=torch.int32)
    for b in range(x.B):
        pages = -(-x.lens[b] // x.page)
        n = min(pages_of(pages), p.topk, pages)
        for i in range(p.blocks):
            for h in range(x.Hkv):
                chosen = torch.randperm(pages - 1, generator=g)[:n - 1].sort()[0]
                idx[b, i, h, :n] = torch.cat([chosen, torch.tensor([pages - 1])]).int()
    return idx


def _runs_wide(x, p, listed):
    """Whether bf16 keys of 16 bits go to the kernel for many rows, and the workgroups that the rows of a block go to."""
    G = x.Hq // x.Hkv
    qblock = p.qblock if listed else min(max(1, 128 // G), p.max_q)
    rows = qblock * G
    parts = -(-rows // (64 if rows <= 64 else 128))
    return rows >= 33 and parts * -(-p.max_q // qblock) * x.Hkv * x.B >= 256, parts


def _shares(x, p, listed):
    """Workgroups that a list is dealt to by the kernel for few rows."""
    G = x.Hq // x.Hkv
    qblock = p.qblock if listed else min(max(1, 128 // G), p.max_q)
    rows = qblock * G
    items = -(-rows // (16 if rows <= 16 else 32)) * -(-p.max_q // qblock) * x.Hkv * x.B
    turns = (p.topk if listed else p.max_pages) * (p.page // 16) // 2
    return max(1, min(-(-1024 // items), turns // 8))


FEW = [  # Hq, news, qblock, topk, lens, listed
    (1, 1024, 1, 700, [11503], True),                        # one row a workgroup, no shares
    (1, 520, 1, 1100, [18500], True),                        # two shares of 550 pages
    (32, 1024, 1, 700, [11503], True),                       # 32 rows
]
WHOLE = (128, 300, 1, 1, [8501], False)                      # without lists: 128 rows a block, four workgroups of 32 (16-bit keys: of 128)
KINDS = [(F, 0, 64), (BF, 4, 128), (F, 4, 64)]


@pytest.mark.parametrize("dtype,bits,d,layout", [(*k, f) for k in [(BF, 0, 64), (BF, 0, 128)] + KINDS for f in FEW] + [(*k, WHOLE) for k in KINDS])
def test_few_rows_over_more_pages_than_are_held(layout, dtype, bits, d):
    Hq, news, qblock, topk, lens, listed = layout
    x = Batch(dtype, bits, d, 16, Hq, 1, lens, [news], 51, extra_pages=0)
    p = x.params(qblock=qblock, topk=topk)
    assert not ((dtype, bits) == (BF, 0) and _runs_wide(x, p, listed)[0])
    shares = _shares(x, p, listed)
    assert (topk if listed else x.max_pages) > HELD * shares and (shares == 2) == (news == 520)
    sel = _long_lists(x, p, lambda pages: topk - 3, 4) if listed else None
    o, lse = B.adacluster_block_attn(p, x.q.cuda(), x.cu_q.cuda(), cache=x.cache, sel_idx=None if sel is None else sel.cuda(), **x.where())
    _check(x, p, sel, o, lse, rows=200 if Hq == 1 else 24)


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,lens,news,qblock,topk,listed", [
    (33, 1, [9003], [257], 1, 560, True),
    (64, 1, [8501, 8209], [256, 256], 2, 1, False),
])
def test_many_rows_over_more_pages_than_are_held(Hq, Hkv, lens, news, qblock, topk, listed, d, causal):
    x = Batch(BF, 0, d, 16, Hq, Hkv, lens, news, 52, extra_pages=0)
    p = x.params(qblock=qblock, topk=topk, causal=causal)
    assert _runs_wide(x, p, listed)[0] and -(-min(lens) // 16) > HELD and (topk > HELD or not listed)
    sel = _long_lists(x, p, lambda pages: topk - 3, 5) if listed else None
    o, lse = B.adacluster_block_attn(p, x.q.cuda(), x.cu_q.cuda(), cache=x.cache, sel_idx=None if sel is None else sel.cuda(), **x.where())
    _check(x, p, sel, o, lse, rows=40)


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("dtype,d,Hq", [(BF, 64, 48), (BF, 128, 33), (BF, 128, 40), (F, 64, 8), (BF, 64, 8)])
@pytest.mark.parametrize("listed", [True, False])
def test_gradients_over_more_pages_than_are_held(listed, dtype, d, Hq, causal):
    """Blocks of one token of many heads; the keys are more than the queries."""
    n, nq = 8600, 40
    x = Batch(dtype, 0, d, 16, Hq, 1, [n], [nq], 53, paged=False, extra_pages=0)
    p = x.params(qblock=1, topk=530, causal=causal)
    assert p.topk > HELD and x.max_pages > HELD
    sel = _long_lists(x, p, lambda pages: 525, 6) if listed else None
    dev = None if sel is None else sel.cuda()
    q, k, v, cu_q, cu_k = x.q.cuda(), x.k.cuda(), x.v.cuda(), x.cu_q.cuda(), x.cu_k.cuda()
    o, lse = B.adacluster_block_attn(p, q, cu_q, k=k, v=v, cu_k=cu_k, sel_idx=dev)
    _check(x, p, sel, o, lse)
    _gradients(x, p, sel, o, lse)


def _gradients(x, p, sel, o, lse):
    d_o = torch.randn(x.q.shape, generator=torch.Generator().manual_seed(2)).to(x.dtype)
    cu_q, cu_k = x.cu_q.cuda(), x.cu_k.cuda()
    grads = B.adacluster_block_attn_backward(p, x.q.cuda(), x.k.cuda(), x.v.cuda(), o, lse, d_o.cuda(), cu_q, cu_k,
                                             sel_idx=None if sel is None else sel.cuda())
    for b in range(x.B):
        aq, ak = slice(int(x.cu_q[b]), int(x.cu_q[b + 1])), slice(int(x.cu_k[b]), int(x.cu_k[b + 1]))
        see = _sees(p, None if sel is None else sel[b].cpu(), x.lens[b], x.news[b])
        r = ref.attend(x.seq(x.q, b), x.seq(x.k, b), x.seq(x.v, b), see, 1 / math.sqrt(x.d), x.dtype, d_o=d_o[aq])
        for got, at, name in zip(grads, (aq, ak, ak), ("dq", "dk", "dv")):
            _within(got[at], r[name], r[name + "_tol"], "%s of sequence %d" % (name, b))


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,Hq,Hkv,lens,news,qblock,topk,listed", [
    (32, 64, 8, [200, 160], [160, 150], 20, 5, True),        # 160 rows: 128 and 32
    (128, 64, 8, [515, 300], [515, 256], 100, 3, True),      # 800 rows: the last of seven workgroups has one wave
    (64, 130, 1, [300], [128], 1, 1, False),                 # 130 heads of one token: 128 and two
    (16, 33, 8, [290, 100, 40], [290, 100, 60], 8, 7, True), # 33 heads are no multiple of anything, and 264 rows: 128, 128 and 8
])
def test_the_rows_of_a_block_over_several_workgroups(page, Hq, Hkv, lens, news, qblock, topk, listed, d, causal):
    if Hq == 33:
        Hq *= Hkv
    x = Batch(BF, 0, d, page, Hq, Hkv, lens, news, 54)
    p = x.params(qblock=qblock, topk=topk, causal=causal)
    wide, parts = _runs_wide(x, p, listed)
    assert wide and parts > 1 and qblock * Hq // Hkv % 128
    q, cu_q = x.q.cuda(), x.cu_q.cuda()
    sel = B.adacluster_block_select(p, q, cu_q, x.cache.boxes, **x.where())[0] if listed else None
    o, lse = B.adacluster_block_attn(p, q, cu_q, cache=x.cache, sel_idx=sel, **x.where())
    _check(x, p, sel, o, lse, rows=60)


@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("d,page,Hq,Hkv,lens,qblock,topk,causal", [
    (64, 64, 8, 1, [333], 20, 4, 1),                         # 160 rows: 128 and 32 (d = 128: 64, 64 and 32)
    (64, 128, 12, 2, [400, 77], 33, 3, 0),                   # 198 rows
    (128, 64, 8, 1, [333], 20, 4, 1),
    (128, 128, 12, 2, [400, 77], 33, 3, 0),
    (64, 64, 130, 1, [70], 1, 2, 1),                         # 130 heads of one token, without lists too
    (128, 64, 130, 1, [70], 1, 2, 1),
])
def test_gradients_of_blocks_over_several_workgroups(d, page, Hq, Hkv, lens, qblock, topk, causal, listed):
    x = Batch(BF, 0, d, page, Hq, Hkv, lens, lens, 55, paged=False)
    p = x.params(qblock=qblock, topk=topk, causal=causal)
    q, k, v, cu_q, cu_k = x.q.cuda(), x.k.cuda(), x.v.cuda(), x.cu_q.cuda(), x.cu_k.cuda()
    sel = B.adacluster_block_select(p, q, cu_q, B.adacluster_block_boxes(p, k, cu_k), cu_k=cu_k)[0] if listed else None
    o, lse = B.adacluster_block_attn(p, q, cu_q, k=k, v=v, cu_k=cu_k, sel_idx=sel)
    _check(x, p, sel, o, lse)
    _gradients(x, p, sel, o, lse)
