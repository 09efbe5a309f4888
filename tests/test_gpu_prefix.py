"""Attention over a cache whose sequences share prefixes (adacluster_prefix_attn) against its definition in 64 bits: one query a
sequence and many, groups of one row and of thousands, prefixes of nothing, that end inside a page, and that some queries or
sequences end in, 16, 32 and 4 bits.  Bounds are those of tests/block_reference.py: the same products, in another order."""
import math
from dataclasses import replace

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within

pytestmark = pytest.mark.gpu


class Shared:
    """A Batch whose groups cu_group share prefix[g] positions.  Rows of page_table of all but a group's first sequence name nothing there."""

    def __init__(self, x, cu_group, prefix, name_pages=False):
        self.x, self.cu_group, self.prefix = x, cu_group, prefix
        self.table = x.table.clone()
        self.whole = [0] * x.B                                   # positions that come from the first sequence `of`
        self.of = list(range(x.B))
        for g, p in enumerate(prefix):
            a, z = cu_group[g], cu_group[g + 1]
            for b in range(a, z):
                self.whole[b] = max(0, min(p, x.lens[a], x.max_pages * x.page)) // x.page * x.page
                self.of[b] = a
                if b > a:
                    self.table[b, :self.whole[b] // x.page] = x.table[a, :self.whole[b] // x.page] if name_pages else -1

    def keys(self, b):
        """k, v in 64 bits and what enters the products"""
        first, own = self.x.keys(self.of[b]), self.x.keys(b)
        w, n = self.whole[b], self.x.lens[b]
        return [None if y is None else torch.cat([f[:w], y[w:]])[:n] for f, y in zip(first, own)]

    def ints(self):
        x = self.x
        return dict(seq_lens=x.lens_t.cuda(), page_table=self.table.cuda(), cu_group=torch.tensor(self.cu_group, dtype=torch.int32).cuda(),
                    prefix_lens=torch.tensor(self.prefix, dtype=torch.int32).cuda())

    def check(self, p, o, lse, scale=None, max_q=None):
        x = self.x
        for b in range(x.B):
            n, nq = x.lens[b], x.news[b]
            k, v, ka, va = self.keys(b)
            see = torch.ones((nq, n), dtype=torch.bool)
            if p.causal:
                see = torch.arange(n) <= n - nq + torch.arange(nq)[:, None]
            r = ref.attend(x.seq(x.q, b), k, v, see[:, None].expand(-1, x.Hkv, -1), scale or 1 / math.sqrt(x.d), x.dtype, ka, va)
            m = min(nq, max_q or nq)
            at = slice(int(x.cu_q[b]), int(x.cu_q[b]) + m)
            _within(o[at], r["o"][:m], r["o_tol"][:m], "o of sequence %d" % b)
            _within(lse[at], r["lse"][:m], r["lse_tol"][:m], "lse of sequence %d" % b)


LAYOUTS = [  # d, page, Hq, Hkv, lens, news, cu_group, prefix
    (64, 16, 4, 4, [1], [1], [0, 1], [1]),
    (64, 16, 8, 8, [100, 77, 65, 90], [1, 1, 1, 1], [0, 4], [64]),
    (128, 16, 8, 2, [333, 300, 290, 1, 40], [1, 1, 1, 1, 1], [0, 3, 5], [289, 1]),                  # (the last group: no whole page)
    (128, 32, 12, 4, [700, 641, 641, 900, 650], [1, 1, 0, 1, 1], [0, 3, 3, 5], [640, 5, 641]),       # an empty group, a sequence without a query
    (64, 64, 6, 2, [500, 0, 450, 131], [1, 1, 1, 1], [1, 2, 4], [300, 130]),                        # a sequence outside, one without keys
    (64, 16, 15, 3, [200, 180, 170], [5, 3, 4], [0, 3], [167]),                                     # some queries end in the prefix
    (128, 16, 5, 1, [90, 40, 60], [5, 5, 3], [0, 3], [85]),                                         # a sequence ends in it
    (64, 32, 3, 3, [40, 33], [50, 40], [0, 2], [32]),                                               # more queries than positions
    (128, 128, 8, 8, [300, 290, 400, 380], [1, 2, 1, 1], [0, 2, 4], [256, 300]),
    (64, 16, 1, 1, [5000, 4900, 4801], [1, 1, 1], [0, 3], [4800]),                                  # few rows: the prefix in many shares
    (128, 64, 16, 2, [3000, 2900], [1, 1], [0, 0, 2], [7, 2890]),
    (64, 16, 4, 2, [100, 90], [1, 1], [0], []),                                                     # no groups
    (64, 16, 64, 1, [300, 280], [1, 1], [0, 2], [270]),                                             # 64 heads a head of keys
    (128, 16, 150, 1, [150, 140, 20], [2, 1, 1], [0, 3], [130]),                                    # and 150
]
WIDE = [  # launches of the kernel for many rows (16 bits), sequences of any number of queries behind them
    (64, 16, 8, 1, [500 + i for i in range(12)], [1] * 12, [0, 5, 12], [480, 333]),
    (128, 16, 16, 4, [900 + 3 * i for i in range(40)], [1] * 40, [0, 17, 40], [890, 801]),
    (128, 64, 4, 4, [300] * 50, [1] * 50, [0, 50], [256]),
    (64, 128, 6, 2, [700 - i for i in range(30)], [1 + i % 5 for i in range(30)], [0, 20, 21, 30], [680, 600, 670]),
    (128, 32, 8, 2, [400, 380, 401], [60, 80, 33], [0, 3], [352]),                                  # queries that the prefix cuts
    (64, 64, 2, 1, [520, 530], [200, 300], [0, 2], [320]),
    (128, 16, 8, 8, [9000, 8990] + [8900] * 40, [1] * 42, [0, 42], [8880]),                         # more than 512 pages a share and few
    (64, 16, 8, 1, [1500 + 7 * i for i in range(12)], [1] * 12, [0, 5, 12], [1480, 1333]),          # 4 bits: tiles of 64 rows
    (64, 64, 12, 1, [1400 + i for i in range(12)], [1] * 12, [0, 12], [1399]),                      # and of 128, own rows few
]


def _run(layout, dtype, bits, causal, name_pages=False, **kw):
    d, page, Hq, Hkv, lens, news, cu_group, prefix = layout
    x = Batch(dtype, bits, d, page, Hq, Hkv, lens, news, 9)
    s = Shared(x, cu_group, prefix, name_pages)
    p = x.params(causal=causal, **kw)
    q = x.q.cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0], Hq), 7.0, device="cuda")
    o, l = B.adacluster_prefix_attn(p, q, x.cu_q.cuda(), x.cache, **s.ints(), out=out, lse=lse)
    s.check(p, o, l)
    rest = int(x.cu_q[-1])
    assert bool((o[rest:] == 7).all()) and bool((l[rest:] == 7).all())


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4), (F, 4)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_shared_prefixes(layout, dtype, bits, causal):
    _run(layout, dtype, bits, causal)


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4)])
@pytest.mark.parametrize("layout", WIDE)
def test_shared_prefixes_of_many_rows(layout, dtype, bits, causal):
    _run(layout, dtype, bits, causal, name_pages=True)


@pytest.mark.parametrize("scale", [1e-3, 0.7, 3.0])
def test_scales(scale):
    x = Batch(BF, 0, 64, 16, 8, 2, [300, 280, 270], [1, 1, 1], 4)
    s = Shared(x, [0, 3], [260])
    p = x.params(softmax_scale=scale)
    o, lse = B.adacluster_prefix_attn(p, x.q.cuda(), x.cu_q.cuda(), x.cache, **s.ints())
    s.check(p, o, lse, scale)


@pytest.mark.parametrize("dtype", [BF, F])
def test_queries_past_max_q_are_left_as_they_were(dtype):
    for Hq, Hkv in ((4, 2), (40, 1)):
        x = Batch(dtype, 0, 64, 16, Hq, Hkv, [200, 190, 180], [6, 2, 5], 4)
        s = Shared(x, [0, 3], [170])
        p = replace(x.params(), max_q=3)
        q = x.q.cuda()
        out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0], Hq), 7.0, device="cuda")
        B.adacluster_prefix_attn(p, q, x.cu_q.cuda(), x.cache, **s.ints(), out=out, lse=lse)
        s.check(p, out, lse, max_q=3)
        for b, nq in enumerate(x.news):
            at = slice(int(x.cu_q[b]) + min(nq, 3), int(x.cu_q[b + 1]))
            assert bool((out[at] == 7).all()) and bool((lse[at] == 7).all())


@pytest.mark.parametrize("dtype", [BF, F])
def test_strides(dtype):
    """Rows of q and o inside wider rows, heads first, and a pool whose heads lie behind each other's pages."""
    x = Batch(dtype, 0, 64, 16, 8, 2, [200 + i for i in range(12)], [1 + i % 3 for i in range(12)], 4)
    s = Shared(x, [0, 7, 12], [190, 100])
    p = x.params()
    heads_first = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    pool = lambda t: t.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3)  # noqa: E731
    q = x.q.cuda()
    wide = torch.zeros((q.shape[0], 9, 80), dtype=dtype, device="cuda")
    wide[:, 1:, 8:72] = q
    cache = replace(x.cache, k=pool(x.cache.k), v=pool(x.cache.v))
    base = B.adacluster_prefix_attn(p, q, x.cu_q.cuda(), x.cache, **s.ints())
    for qq, out in ((heads_first(q), None), (wide[:, 1:, 8:72], torch.zeros_like(wide)[:, 1:, 8:72])):
        o, lse = B.adacluster_prefix_attn(p, qq, x.cu_q.cuda(), cache, **s.ints(), out=out)
        s.check(p, o, lse)
        n = int(x.cu_q[-1])
        assert torch.equal(o[:n], base[0][:n]) and torch.equal(lse[:n], base[1][:n])


@pytest.mark.parametrize("news", [[1] * 12, [7] * 12])
def test_tokens_of_a_page_far_apart(news):
    """Strides of a pool past what 32 bits of an offset hold: the kernel for few rows takes any number of them."""
    x = Batch(BF, 0, 64, 16, 8, 2, [200 + i for i in range(12)], news, 4)
    s = Shared(x, [0, 7, 12], [190, 100])
    n = x.cache.k.shape[0]
    far = torch.empty(16 << 25, dtype=BF, device="cuda")
    pool = [far.as_strided((n, 2, 16, 64), (128, 64, 1 << 25, 1), at) for at in (0, 1 << 24)]
    for to, of in zip(pool, (x.cache.k, x.cache.v)):
        to.copy_(of)
    o, lse = B.adacluster_prefix_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), replace(x.cache, k=pool[0], v=pool[1]), **s.ints())
    s.check(x.params(), o, lse)


def test_pages_that_name_nothing_and_wild_device_data():
    """Entries outside the pool name no keys, in the prefix and behind it; lengths and groups are held to the buffers."""
    x = Batch(BF, 0, 64, 16, 4, 2, [160, 150, 140], [1, 1, 1], 4)
    s = Shared(x, [0, 3], [96])
    gone = dict(s.ints())
    table = s.table.clone()
    table[0, 2], table[1, 7], table[2, 6] = -1, 1 << 30, x.cache.k.shape[0]
    gone["page_table"] = table.cuda()
    o, lse = B.adacluster_prefix_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), x.cache, **gone)
    for b, missing in enumerate(([2], [2, 7], [2, 6])):
        k, v, _, _ = s.keys(b)
        there = torch.ones(x.lens[b], dtype=torch.bool)
        for pg in missing:
            there[16 * pg:16 * pg + 16] = False
        r = ref.attend(x.seq(x.q, b), k, v, there[None, None].expand(1, 2, -1), 1 / 8, BF)
        _within(o[b:b + 1], r["o"], r["o_tol"], "o")
        _within(lse[b:b + 1], r["lse"], r["lse_tol"], "lse")
    wild = s.ints()
    for name, value in (("cu_group", [-5, 1 << 30]), ("cu_group", [3, 0]), ("prefix_lens", [1 << 30]), ("prefix_lens", [-(1 << 31)]),
                        ("seq_lens", [1 << 30, -7, 50])):
        bad = dict(wild)
        bad[name] = torch.tensor(value, dtype=torch.int64).to(torch.int32).cuda()
        B.adacluster_prefix_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), x.cache, **bad)
    for cu in ([0, 1 << 30, -3, 2], [9, 9, 9, 9], [3, 2, 1, 0]):
        B.adacluster_prefix_attn(x.params(), x.q.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), x.cache, **wild)
    torch.cuda.synchronize()


def test_rows_behind_the_last_sequence_by_far():
    """A buffer of queries for far more than the call's: its size bounds the shares, not the results."""
    x = Batch(BF, 0, 64, 16, 8, 2, [300, 290], [1, 1], 4, spare=200000)
    s = Shared(x, [0, 2], [280])
    out = torch.full_like(x.q, 7.0, device="cuda")
    o, lse = B.adacluster_prefix_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), x.cache, **s.ints(), out=out)
    s.check(x.params(), o, lse)
    assert bool((o[2:] == 7).all())


def test_a_call_on_tensors_that_require_gradients_warns():
    x = Batch(BF, 0, 64, 16, 2, 2, [40, 40], [1, 1], 4)
    s = Shared(x, [0, 2], [32])
    with pytest.warns(UserWarning, match="records nothing"):
        _, lse = B.adacluster_prefix_attn(x.params(), x.q.cuda().requires_grad_(), x.cu_q.cuda(), x.cache, **s.ints())
    with pytest.warns(UserWarning, match="records nothing"):
        w = B.adacluster_cache_weights(x.params(), x.q.cuda().requires_grad_(), x.cu_q.cuda(), lse, x.cache, **x.where())
    assert not lse.requires_grad and not w.requires_grad


@pytest.mark.parametrize("rows_heads", [(4, 2), (64, 2)])
def test_infinities_behind_the_end_and_scores_of_minus_infinity(rows_heads):
    """A key whose score is -inf weighs nothing; a row that sees no other is empty.  The pool is NaN wherever no key lies."""
    Hq, Hkv = rows_heads
    x = Batch(BF, 0, 64, 16, Hq, Hkv, [40, 33], [1, 1], 4)
    s = Shared(x, [0, 2], [32])
    k = x.cache.k
    k[x.table[0, :3].long().cuda()] = -math.inf
    k[x.table[1, 2].long().cuda()] = -math.inf
    q = x.q.abs().cuda() + 0.5
    o, lse = B.adacluster_prefix_attn(x.params(), q, x.cu_q.cuda(), x.cache, **s.ints())
    assert bool((o[:2] == 0).all()) and bool((lse[:2] == -math.inf).all())


def test_empty_calls_streams_graphs_and_repeats():
    x = Batch(BF, 0, 128, 16, 16, 2, [900 + i for i in range(9)], [1] * 9, 4)
    s = Shared(x, [0, 9], [890])
    p, q, cu = x.params(), x.q.cuda(), x.cu_q.cuda()
    ints = s.ints()
    o, lse = B.adacluster_prefix_attn(p, q[:0], torch.zeros_like(cu), x.cache, **ints)
    assert o.shape == (0, 16, 128) and lse.shape == (0, 16)
    base = B.adacluster_prefix_attn(p, q, cu, x.cache, **ints)
    torch.cuda.synchronize()
    n = int(x.cu_q[-1])
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):                                           # two calls at once
        got = []
        for st in side:
            with torch.cuda.stream(st):
                got.append(B.adacluster_prefix_attn(p, q, cu, x.cache, **ints))
        torch.cuda.synchronize()
        for o, lse in got:
            assert torch.equal(o[:n], base[0][:n]) and torch.equal(lse[:n], base[1][:n])
    graphs, outs, inputs = [], [], [q.clone(), q.clone()]
    for qq in inputs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(B.adacluster_prefix_attn(p, qq, cu, x.cache, **ints))
        graphs.append(g)
    for turn in range(3):
        for i, qq in enumerate(inputs):
            qq.copy_(q * (0.5 + turn + i))
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for qq, (o, lse) in zip(inputs, outs):
            want = B.adacluster_prefix_attn(p, qq, cu, x.cache, **ints)
            torch.cuda.synchronize()
            assert torch.equal(o[:n], want[0][:n]) and torch.equal(lse[:n], want[1][:n])
