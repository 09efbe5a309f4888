"""What the calls over a cache give after an eviction: attention and the pages that blocks select against their definitions in 64 bits, over the tokens that
stayed as they lie in the new pages."""
import math
from dataclasses import replace

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within
from tests.test_gpu_keep import Evicted, _random_weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4)])
@pytest.mark.parametrize("d,page,keep", [(64, 16, 61), (128, 32, 130)])
def test_attention_and_selection_over_what_stayed(dtype, bits, d, page, keep):
    Hq, Hkv = 8, 2
    x = Batch(dtype, bits, d, page, Hq, Hkv, [300, 190, keep - 3], [1, 1, 1], 8)
    p = x.params(keep_first=1)
    q, cu = x.q[:3].cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    w = B.adacluster_cache_weights(p, q, cu, lse, x.cache, **x.where())
    e = Evicted(x, w.cpu(), keep, 9, 1)
    kept, now, _ = e.run(p)
    e.check(kept, now, _)
    c, table = e.cache, e.new_table

    def rows(b, codes, meta):
        """[n, Hkv, d] of sequence b from the pages of the new table, in 64 bits"""
        n = int(now[b])
        at = table[b, :-(-n // page)].long().cuda()
        y = ref.dequantise(codes[at].cpu(), meta[at].cpu()) if bits else codes[at].cpu().double()
        return y.transpose(1, 2).flatten(0, 1)[:n]

    def enters(b, meta):
        n = int(now[b])
        m = meta[table[b, :-(-n // page)].long().cuda()].cpu().double()
        return (143 * m[..., 0] + m[..., 1].abs()).repeat_interleave(64, -1).transpose(1, 2).flatten(0, 1)[:n]

    g = torch.Generator().manual_seed(7)
    q = torch.randn((3, Hq, d), generator=g).to(dtype)
    groups = dict(cu_group=torch.tensor([0, 1, 2, 3], dtype=torch.int32).cuda(), prefix_lens=torch.tensor([keep // 2, 0, keep], dtype=torch.int32).cuda())
    lists = replace(p, keep_first=0, topk=2, qblock=1)
    got = [B.adacluster_block_attn(p, q.cuda(), cu, cache=c, seq_lens=now, page_table=table.cuda()),
           B.adacluster_prefix_attn(p, q.cuda(), cu, c, now, table.cuda(), **groups)]
    sel, cnt = B.adacluster_block_select(lists, q.cuda(), cu, c.boxes, seq_lens=now, page_table=table.cuda())
    listed = B.adacluster_block_attn(lists, q.cuda(), cu, cache=c, seq_lens=now, page_table=table.cuda(), sel_idx=sel)
    others = 0
    for b in range(3):
        n = int(now[b])
        k, v = rows(b, c.k, c.k_meta), rows(b, c.v, c.v_meta)
        ka, va = (enters(b, c.k_meta), enters(b, c.v_meta)) if bits else (None, None)
        boxes = ref.boxes_of(k.to(dtype), page)
        assert torch.equal(c.boxes[table[b, :-(-n // page)].long().cuda()].cpu(), boxes)
        want = ref.select(q[b:b + 1], boxes, n, 1, Hkv, page, 1, 2, 0, 1)
        mine = [[[y for y in sel[b, 0, h].tolist() if y >= 0] for h in range(Hkv)]]
        assert mine == want, b
        others += sum(0 not in y for y in want[0])
        every = torch.ones((1, Hkv, n), dtype=torch.bool)
        for (o, l), see in ((got[0], every), (got[1], every), (listed, ref.sees(want, n, 1, Hkv, page, 1, 1))):
            r = ref.attend(q[b:b + 1], k, v, see, 1 / math.sqrt(d), dtype, ka, va)
            _within(o[b:b + 1], r["o"], r["o_tol"], "o of sequence %d" % b)
            _within(l[b:b + 1], r["lse"], r["lse_tol"], "lse of sequence %d" % b)
    assert others                                                # some lists leave the first page out


@pytest.mark.parametrize("kind", ["plain", "ties"])
def test_a_second_eviction(kind):
    """From the new pages on, with the weights that came along, to the pages that the first one gave away."""
    x = Batch(BF, 0, 64, 16, 4, 2, [300, 150, 60], [0, 0, 0], 8)
    p = x.params(keep_first=1)
    e = Evicted(x, _random_weights(x, kind, 2), 100, 9, 1)
    kept, now, w = e.run(p)
    e.check(kept, now, w)
    old = x.table.clone()
    k0, v0 = e.cache.k.cpu(), e.cache.v.cpu()
    to = torch.full_like(old, -1)
    to[:, :4] = old[:, :4]
    kept2, now2, w2 = B.adacluster_cache_evict(p, e.cache, now, e.new_table.cuda(), w, 50, 5, to.cuda())
    assert now2.tolist() == [50, 50, 50]
    for b in range(3):
        for h in range(2):
            n = int(now[b])
            ws = w[b, h, :n].tolist()
            must = set(range(16)) | set(range(n - 5, n))
            rest = sorted((j for j in range(n) if j not in must), key=lambda j: (-ws[j], j))
            stay = sorted(must | set(rest[:50 - len(must)]))
            assert kept2[b, h].tolist() == stay and w2[b, h, :50].tolist() == [ws[j] + 0.0 for j in stay]
            for i, j in enumerate(stay):
                a, z = (int(to[b, i // 16]), i % 16), (int(e.new_table[b, j // 16]), j % 16)
                for new, before in ((e.cache.k, k0), (e.cache.v, v0)):
                    assert torch.equal(new[a[0], h, a[1]].cpu(), before[z[0], h, z[1]])
