"""What a sequence keeps of its cache: weights of cached keys (adacluster_cache_weights) against their definition in 64 bits, the tokens
that stay and their move (adacluster_cache_evict) exactly, and a run of all calls together.

Bound of a weight: every term p = exp(s - lse) is off by the error of its score, es = (d + 8) u scale sum |q||k| (the bound of
tests/block_reference.py), by the roundings of scale * log2(e), lse * log2(e) and their difference (4 u (|s| + |lse|)) and of the exponential (8 u);
n terms are summed in fp32 in some order ((n + 64) u of the sum), and the weight before is multiplied and added (2 u)."""
import math
from dataclasses import replace

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within
from tests.test_gpu_prefix import Shared

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _weights(x, b, lse, scale, causal, before, there=None):
    """weights [Hkv, n] of sequence b in 64 bits and their bound"""
    n, nq, G = x.lens[b], x.news[b], x.Hq // x.Hkv
    k, _, ka, _ = x.keys(b)
    k = k.double()
    ka = k.abs() if ka is None else ka
    q = x.seq(x.q, b).double()
    see = torch.ones((nq, n), dtype=torch.bool)
    if causal:
        see = torch.arange(n) <= n - nq + torch.arange(nq)[:, None]
    if there is not None:
        see = see & there
    w = torch.zeros((x.Hkv, n), dtype=torch.float64)
    tol = torch.zeros_like(w)
    for h in range(x.Hq):
        l = lse[int(x.cu_q[b]):int(x.cu_q[b + 1]), h].double()[:, None]
        s = scale * q[:, h] @ k[:, h // G].T
        es = (x.d + 8) * U * scale * (q[:, h].abs() @ ka[:, h // G].T)
        live = see & (l > -math.inf)
        e = torch.where(live, (s - torch.where(l > -math.inf, l, 0.0)).exp(), 0.0)
        w[h // G] += e.sum(0)
        tol[h // G] += torch.where(live, e * (es + 4 * U * (s.abs() + l.abs()) + 8 * U), 0.0).sum(0) * 1.02
    tol += (nq * G + 64) * U * w
    if before is not None:
        w = w + before
        tol = tol + 2 * U * (w.abs() + before.abs())
    return w, tol


LAYOUTS = [  # d, page, Hq, Hkv, lens, news
    (64, 16, 4, 4, [1], [1]),
    (128, 16, 8, 2, [333, 0, 129, 16], [1, 1, 1, 1]),
    (64, 32, 6, 2, [95, 31, 130], [1, 0, 1]),
    (128, 64, 5, 1, [257, 64, 1], [7, 3, 1]),
    (64, 128, 3, 3, [300, 129], [300, 40]),
    (128, 32, 2, 2, [90, 40], [20, 60]),                          # more queries than positions
    (64, 16, 40, 2, [211], [100]),
    (128, 16, 32, 8, [700, 650], [64, 33]),
    (64, 64, 64, 1, [500], [3]),
    (128, 128, 12, 4, [1000, 999], [257, 129]),
    (64, 16, 8, 1, [300], [290]),                                 # (16 bits: few keys for many rows, which are shared out)
    (128, 32, 15, 3, [200, 7, 90], [200, 1, 90]),
    (64, 16, 96, 1, [130, 40], [3, 2]),                           # more heads a key than rows a stage
    (128, 16, 200, 2, [100], [7]),
]


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4), (F, 4)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_weights(layout, dtype, bits, causal):
    d, page, Hq, Hkv, lens, news = layout
    x = Batch(dtype, bits, d, page, Hq, Hkv, lens, news, 6)
    p = x.params(causal=causal)
    q, cu = x.q.cuda(), x.cu_q.cuda()
    lse = torch.full((q.shape[0], Hq), math.nan, device="cuda")
    B.adacluster_block_attn(p, q, cu, cache=x.cache, lse=lse, **x.where())
    shape = (x.B, Hkv, x.max_pages * page)
    g = torch.Generator().manual_seed(2)
    before = torch.rand(shape, generator=g)
    for b, n in enumerate(lens):
        before[b, :, n:] = math.nan                               # nobody's
    lse_host = lse.cpu()
    for decay, w in ((1.0, None), (0.0, torch.full(shape, math.nan)), (0.75, before), (1.0, before)):
        got = B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=None if w is None else w.cuda(), decay=decay, **x.where())
        for b, n in enumerate(lens):
            want, tol = _weights(x, b, lse_host, 1 / math.sqrt(d), causal, decay * w[b, :, :n].double() if w is not None and decay else None)
            _within(got[b, :, :n], want, tol, "weights of sequence %d, decay %g" % (b, decay))
            assert bool((got[b, :, n:] == 0).all())
    # in place, and without an earlier weight: every row's weights sum to one
    w = before.cuda()
    out = B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.75, out=w, **x.where())
    assert out is w
    ones = B.adacluster_cache_weights(p, q, cu, lse, x.cache, decay=0.0, weights=w, **x.where())
    for b in range(x.B):
        rows = lse_host[int(x.cu_q[b]):int(x.cu_q[b + 1])]
        for h in range(Hkv):
            count = int((rows[:, h * (Hq // Hkv):(h + 1) * (Hq // Hkv)] > -math.inf).sum())
            assert abs(float(ones[b, h].double().sum()) - count) <= 1e-3 * max(1, count)


@pytest.mark.parametrize("bits,news", [(0, 1), (4, 1), (0, 40), (4, 40)])
def test_weights_in_a_graph_and_on_two_streams(bits, news):
    x = Batch(BF, bits, 64, 16, 8, 2, [300, 200], [news, news], 6)
    p, q, cu = x.params(), x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    w = torch.rand((2, 2, x.max_pages * 16), device="cuda")
    where = x.where()
    base = B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.5, **where)
    torch.cuda.synchronize()
    side, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for st in side:
        with torch.cuda.stream(st):
            got.append(B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.5, **where))
    torch.cuda.synchronize()
    assert all(torch.equal(base, y) for y in got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.5, **where)
    for turn in range(3):
        w.copy_(torch.rand(w.shape, generator=torch.Generator().manual_seed(turn)))
        q.copy_(x.q * (1 + turn))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.5, **where)
        assert torch.equal(out, want)


def test_weights_of_heads_far_apart():
    """Heads of a query too far apart for the offsets of the kernel for many rows (and near enough): the same weights."""
    x = Batch(BF, 0, 64, 16, 4, 1, [100], [12], 6)
    p, q, cu = x.params(), x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    want, tol = _weights(x, 0, lse.cpu(), 1 / 8, 1, None)
    for stride in (1 << 20, 1 << 29):
        far = torch.empty(3 * stride + q.shape[0] * 64, dtype=BF, device="cuda")
        view = far.as_strided(q.shape, (64, stride, 1))
        view.copy_(q)
        got = B.adacluster_cache_weights(p, view, cu, lse, x.cache, **x.where())
        _within(got[0, :, :100], want, tol, "weights, heads %d apart" % stride)


def test_weights_of_many_rows_in_place_equal_those_apart():
    x = Batch(BF, 0, 128, 16, 16, 4, [600, 500], [100, 70], 6)
    p = x.params()
    q, cu = x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    w = torch.rand((2, 4, x.max_pages * 16), device="cuda")
    apart = B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.5, **x.where())
    B.adacluster_cache_weights(p, q, cu, lse, x.cache, weights=w, decay=0.5, out=w, **x.where())
    assert torch.equal(apart, w)


@pytest.mark.parametrize("news", [1, 8, 40, 100])
def test_weights_of_scores_that_no_query_makes(news):
    """The last key is infinite: the only query that sees it scores -inf, all others +inf, and rows behind the last one score nothing."""
    x = Batch(BF, 0, 64, 16, 2, 2, [130], [news], 6)
    x.q = x.q.abs() + 0.1
    x.q[news - 1] *= -1
    at = 129
    x.cache.k[int(x.table[0, at // 16]), :, at % 16] = math.inf
    p = x.params()
    q, cu = x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    got = B.adacluster_cache_weights(p, q, cu, lse, x.cache, **x.where())
    want, tol = _weights(x, 0, lse.cpu(), 1 / 8, 1, None, torch.arange(130) < at)
    _within(got[0, :, :at], want[:, :at], tol[:, :at], "weights")
    assert bool((got[0, :, at:] == 0).all())


@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4), (F, 4)])
def test_weights_at_the_edges(dtype, bits):
    """lse of -inf adds nothing, pages that are not named and queries past max_q neither; strides; a step without queries."""
    x = Batch(dtype, bits, 64, 16, 4, 2, [100, 90], [5, 4], 6)
    p = x.params()
    q, cu = x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    lse[1] = -math.inf
    lse[6, 2] = -math.inf
    where = x.where()
    table = x.table.clone()
    table[0, 3], table[1, 0] = -1, 1 << 30
    where["page_table"] = table.cuda()
    wide = torch.zeros((q.shape[0], 5, 80), dtype=dtype, device="cuda")
    wide[:, 1:, 8:72] = q
    there = [torch.ones(n, dtype=torch.bool) for n in x.lens]
    there[0][48:64] = False
    there[1][:16] = False
    base = None
    for qq in (q, wide[:, 1:, 8:72], q.transpose(0, 1).contiguous().transpose(0, 1)):
        got = B.adacluster_cache_weights(p, qq, cu, lse, x.cache, **where)
        for b, n in enumerate(x.lens):
            want, tol = _weights(x, b, lse.cpu(), 1 / 8, 1, None, there[b])
            _within(got[b, :, :n], want, tol, "weights of sequence %d" % b)
            assert bool((got[b, :, :n][:, ~there[b]] == 0).all())
        assert base is None or torch.equal(base, got)
        base = got
    short = replace(p, max_q=2)
    got = B.adacluster_cache_weights(short, q, cu, lse, x.cache, **x.where())
    cut = lse.clone()
    cut[2:5] = cut[7:9] = -math.inf
    want = B.adacluster_cache_weights(p, q, cu, cut, x.cache, **x.where())
    for b, n in enumerate(x.lens):
        w, tol = _weights(x, b, cut.cpu(), 1 / 8, 1, None)
        _within(got[b, :, :n], w, tol, "two queries of sequence %d" % b)
        _within(want[b, :, :n], w, tol, "two queries of sequence %d" % b)
    w = torch.rand(got.shape, device="cuda")
    none = B.adacluster_cache_weights(p, q[:0], torch.zeros_like(cu), lse[:0], x.cache, weights=w, decay=0.5, **x.where())
    for b, n in enumerate(x.lens):
        assert torch.equal(none[b, :, :n], 0.5 * w[b, :, :n]) and bool((none[b, :, n:] == 0).all())
    for cu_bad, lens_bad in (([0, 1 << 30, -3], [100, 90]), ([9, 9, 9], [100, 90]), ([0, 5, 9], [1 << 30, -9])):
        B.adacluster_cache_weights(p, q, torch.tensor(cu_bad, dtype=torch.int32).cuda(), lse, x.cache,
                                   torch.tensor(lens_bad, dtype=torch.int32).cuda(), x.where()["page_table"])
    torch.cuda.synchronize()


# ---- eviction -----------------------------------------------------------------------------------------------------------


def _chosen(w, n, keep, first, recent):
    """Positions that stay of one head, by the definition: w a list of floats."""
    if n <= keep:
        return list(range(n))
    must = [j for j in range(n) if j < first or j >= n - recent]
    rest = [j for j in range(n) if first <= j < n - recent]
    rest.sort(key=lambda j: (0, -w[j], j) if w[j] == w[j] else (1, 0.0, j))
    return sorted(must + rest[:keep - len(must)])


class Evicted:
    """A Batch with pages to spare, and what the pool is after an eviction, by the definition."""

    def __init__(self, x, weights, keep, recent, first, same=(), seed=3):
        g = torch.Generator().manual_seed(seed)
        self.x, self.w, self.keep, self.recent, self.first = x, weights, keep, recent, first
        c, old = x.cache, x.cache.k.shape[0]
        per = [-(-min(n, keep) // x.page) for n in x.lens]
        spare = sum(per) + 2
        grow = lambda t: None if t is None else torch.cat([t, torch.randint(0, 256, (spare, *t.shape[1:]), generator=g).to(t.dtype).cuda()])  # noqa: E731
        self.cache = B.BlockCache(*[grow(t) for t in (c.k, c.v, c.k_meta, c.v_meta, c.boxes)])
        order = old + torch.randperm(spare, generator=g).int()
        self.new_table = torch.full((x.B, x.max_pages), -1, dtype=torch.int32)
        at = 0
        for b, k in enumerate(per):
            self.new_table[b, :k] = order[at:at + k]
            at += k
        for b, pages in same:                                     # pages that stay in their place
            self.new_table[b, :pages] = x.table[b, :pages]
        self.before = [None if t is None else t.clone() for t in (self.cache.k, self.cache.v, self.cache.k_meta, self.cache.v_meta, self.cache.boxes)]

    def run(self, p, **kw):
        x = self.x
        return B.adacluster_cache_evict(p, self.cache, x.lens_t.cuda(), x.table.cuda(), self.w.cuda(), self.keep, self.recent, self.new_table.cuda(), **kw)

    def check(self, kept, lens, new_w):
        x, page = self.x, self.x.page
        want = [None if t is None else t.cpu() for t in self.before]
        parts = want[:2] if x.bits == 0 else want[:4]
        for b, n in enumerate(x.lens):
            m = min(n, self.keep)
            assert int(lens[b]) == m
            for g in range(x.Hkv):
                stay = _chosen(self.w[b, g].tolist(), n, self.keep, self.first * page, self.recent)
                assert kept[b, g].tolist() == stay + [-1] * (self.keep - m), (b, g)
                full = torch.zeros_like(self.w[b, g])
                full[:m] = self.w[b, g, stay]
                got = new_w[b, g].cpu()
                assert torch.equal(got.isnan(), full.isnan()) and torch.equal(got.nan_to_num(7.0), full.nan_to_num(7.0)), (b, g)
                for pg in range(-(-m // page)):
                    to, here = int(self.new_table[b, pg]), stay[pg * page:(pg + 1) * page]
                    if not 0 <= to < want[0].shape[0] or to == int(x.table[b, pg]):
                        continue
                    rows = [(int(x.table[b, j // page]), j % page) for j in here]
                    for t, old in zip(parts, self.before):
                        for i, (a, s) in enumerate(rows):
                            t[to, g, i] = old[a, g, s].cpu() if 0 <= a < old.shape[0] else 0
                    k = want[0][to, g, :len(here)]
                    if x.bits == 4:
                        k = ref.dequantise(k, want[2][to, g, :len(here)]).to(x.dtype)
                    want[4][to, g] = torch.stack([k.amax(0), k.amin(0)])
        raw = lambda t: t.cpu().contiguous().view(torch.uint8)  # noqa: E731
        for name, t, w in zip(("k", "v", "k_meta", "v_meta"), (self.cache.k, self.cache.v, self.cache.k_meta, self.cache.v_meta), want):
            assert t is None or torch.equal(raw(t), raw(w)), name
        assert torch.equal(self.cache.boxes.cpu(), want[4])


EVICT = [  # d, page, Hq, Hkv, lens, keep, recent, first
    (64, 16, 4, 4, [1], 1, 0, 0),
    (64, 16, 2, 2, [5], 1, 1, 0),
    (128, 16, 8, 2, [100, 40, 33, 0, 17], 33, 5, 1),
    (64, 32, 3, 3, [200, 64, 65], 64, 0, 2),
    (128, 64, 4, 1, [500, 130], 129, 64, 1),
    (64, 128, 2, 2, [700, 90], 300, 44, 2),                       # room for nothing but the first and the last
    (64, 16, 1, 1, [5000, 4097], 1000, 100, 1),                   # more positions than a workgroup takes at a time
    (128, 32, 2, 2, [9000], 8999, 3, 0),
    (64, 16, 2, 1, [300], 5000, 20, 3),                           # more room than there is
    (64, 64, 1, 1, [70001], 40000, 500, 2),                       # three times as many as fit the registers
    (64, 128, 1, 1, [66000, 32768], 32768, 0, 0),
]


def _random_weights(x, kind, seed):
    g = torch.Generator().manual_seed(seed)
    shape = (x.B, x.Hkv, x.max_pages * x.page)
    if kind == "ties":                                            # few values, both zeros, negative ones
        return torch.tensor([0.0, -0.0, 1.0, 2.0, -1.0])[torch.randint(0, 5, shape, generator=g)]
    if kind == "wild":
        w = torch.randn(shape, generator=g) * 10.0 ** torch.randint(-44, 38, shape, generator=g)
        for v in (math.nan, math.inf, -math.inf, -math.nan):
            w[torch.rand(shape, generator=g) < 0.1] = v
        return w
    if kind == "near":                                            # apart by the last bits
        return 1 + torch.randint(0, 40, shape, generator=g) * 2.0 ** -23
    return torch.exp(2 * torch.randn(shape, generator=g))


@pytest.mark.parametrize("kind", ["plain", "ties", "near", "wild"])
@pytest.mark.parametrize("layout", EVICT)
def test_tokens_that_stay(layout, kind):
    d, page, Hq, Hkv, lens, keep, recent, first = layout
    x = Batch(BF, 0, d, page, Hq, Hkv, lens, [0] * len(lens), 8)
    e = Evicted(x, _random_weights(x, kind, 1), keep, recent, first)
    e.check(*e.run(x.params(keep_first=first)))


@pytest.mark.parametrize("dtype,bits", [(F, 0), (BF, 4), (F, 4)])
@pytest.mark.parametrize("layout", EVICT[:6])
def test_moves_of_every_kind_of_cache(layout, dtype, bits):
    d, page, Hq, Hkv, lens, keep, recent, first = layout
    x = Batch(dtype, bits, d, page, Hq, Hkv, lens, [0] * len(lens), 8)
    e = Evicted(x, _random_weights(x, "plain", 2), keep, recent, first)
    e.check(*e.run(x.params(keep_first=first)))


@pytest.mark.parametrize("dtype,d,bits", [(BF, 64, 0), (BF, 128, 4), (F, 64, 0)])
def test_last_pages_of_few_tokens_that_stay(dtype, d, bits):
    """Sequences that keep everything, in their places: pages of any number of tokens are left as they are, their boxes too."""
    lens = [33, 17, 7, 1, 64, 45]
    x = Batch(dtype, bits, d, 16, 2, 2, lens, [0] * 6, 8)
    e = Evicted(x, _random_weights(x, "plain", 2), 64, 4, 1, same=tuple((b, 4) for b in range(6)))
    e.check(*e.run(x.params(keep_first=1)))


@pytest.mark.parametrize("bits", [0, 4])
def test_pages_that_stay_in_their_place(bits):
    """The first pages of a sequence, shared by two of them, and all pages of one that keeps everything; pages that are not named."""
    x = Batch(BF, bits, 64, 16, 4, 2, [200, 100, 60], [0, 0, 0], 8)
    x.table[1, :2] = x.table[0, :2]
    e = Evicted(x, _random_weights(x, "plain", 2), 64, 4, 2, same=((0, 2), (1, 2), (2, 4)))
    e.check(*e.run(x.params(keep_first=2)))
    x = Batch(BF, bits, 64, 16, 4, 2, [200, 100, 60], [0, 0, 0], 8)
    x.table[0, 5], x.table[1, 1] = -1, 1 << 30
    e = Evicted(x, _random_weights(x, "plain", 2), 64, 4, 1)
    e.new_table[0, 1], e.new_table[2, 0] = -1, 1 << 30
    e.check(*e.run(x.params(keep_first=1)))


def test_evict_with_strides_a_graph_and_wild_lengths():
    x = Batch(BF, 0, 64, 16, 4, 2, [300, 150, 60], [0, 0, 0], 8)
    p = x.params(keep_first=1)
    w = _random_weights(x, "ties", 2)
    e = Evicted(x, w, 100, 9, 1)
    pool = lambda t: t.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3)  # noqa: E731
    e.cache = replace(e.cache, k=pool(e.cache.k), v=pool(e.cache.v))
    got = e.run(p)
    e.check(*got)
    args = [e.cache, x.lens_t.cuda(), x.table.cuda(), w.cuda(), 100, 9, e.new_table.cuda()]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = B.adacluster_cache_evict(p, *args)
    for turn in range(3):
        args[3].copy_(_random_weights(x, "plain", turn + 5))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        e.w = args[3].cpu()
        e.check(*out)
        want = B.adacluster_cache_evict(p, *args)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    for lens in ([1 << 30, -5, 60], [0, 0, 0]):
        bad = torch.tensor(lens, dtype=torch.int32).cuda()
        kept, new, _ = B.adacluster_cache_evict(p, e.cache, bad, *args[2:])
        assert new.tolist() == [min(max(0, min(n, x.max_pages * 16)), 100) for n in lens] and int(kept.max()) < x.max_pages * 16


@pytest.mark.parametrize("news", [1, 40])
@pytest.mark.parametrize("dtype,bits,far", [(BF, 0, 66000), (F, 0, 66000), (BF, 4, 265000)])
def test_pools_past_32_bits(dtype, bits, far, news):
    """All calls over a pool whose named pages lie behind 2^32 bytes of others give what they give over the same pages alone."""
    x = Batch(dtype, bits, 128, 128, 4, 2, [300, 290, 140], [news] * 3, 4)
    s, e = Shared(x, [0, 2], [256]), Evicted(x, _random_weights(x, "plain", 2), 150, 20, 1)
    p, q, cu, n = x.params(keep_first=1), x.q.cuda(), x.cu_q.cuda(), 3 * news

    def behind(t):
        if t is not None:
            y = torch.empty((far + t.shape[0], *t.shape[1:]), dtype=t.dtype, device="cuda")
            y[far:] = t
            return y

    def calls(cache, at):
        table = lambda t: torch.where(t >= 0, t + at, t).cuda()  # noqa: E731
        o, lse = B.adacluster_prefix_attn(p, q, cu, cache, **{**s.ints(), "page_table": table(s.table)})
        w = B.adacluster_cache_weights(p, q, cu, lse, cache, x.lens_t.cuda(), table(x.table), e.w.cuda(), 0.5)
        got = B.adacluster_cache_evict(p, cache, x.lens_t.cuda(), table(x.table), w, 150, 20, table(e.new_table))
        return [o[:n], lse[:n], w, *got] + [t[at:] for t in (cache.k, cache.v, cache.k_meta, cache.v_meta, cache.boxes) if t is not None]

    big = calls(B.BlockCache(*[behind(t) for t in (e.cache.k, e.cache.v, e.cache.k_meta, e.cache.v_meta, e.cache.boxes)]), far)
    for i, (a, b) in enumerate(zip(calls(e.cache, 0), big)):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)), i


# ---- together -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4)])
def test_a_server_appends_attends_weighs_and_evicts(dtype, bits):
    """Steps of generation over shared prompts: append, attention with the shared prefix, weights of the keys; then every sequence is cut
    to a budget, keeping the shared pages where they are, and goes on from its new pages.  Attention before and after is that of
    adacluster_block_attn, and attention over what stays that of the definition."""
    d, page, Hq, Hkv, prefix, steps = 64, 16, 8, 2, 48, 5
    lens, news = [80, 70, 75], [1, 1, 1]
    x = Batch(dtype, bits, d, page, Hq, Hkv, lens, news, 13, fill=0.0, extra_pages=2)
    s = Shared(x, [0, 3], [prefix], name_pages=True)
    pool = x.cache.k.shape[0]
    spare = 40
    grow = lambda t: None if t is None else torch.cat([t, torch.zeros((spare, *t.shape[1:]), dtype=t.dtype, device="cuda")])  # noqa: E731
    cache = B.BlockCache(*[grow(t) for t in (x.cache.k, x.cache.v, x.cache.k_meta, x.cache.v_meta, x.cache.boxes)])
    free = list(range(pool, pool + spare))
    table = s.table.clone()
    for b, n in enumerate(lens):
        for pg in range(-(-n // page), x.max_pages):
            table[b, pg] = free.pop()
    table, now = table.cuda(), x.lens_t.cuda()
    cu = torch.arange(4, dtype=torch.int32, device="cuda")
    groups = dict(cu_group=torch.tensor([0, 3], dtype=torch.int32).cuda(), prefix_lens=torch.tensor([prefix], dtype=torch.int32).cuda())
    p = B.BlockParams(B=3, Hq=Hq, Hkv=Hkv, d=d, dtype=B.BF16 if dtype == BF else B.F32, bits=bits, page=page, max_pages=x.max_pages, max_q=1,
                      keep_first=prefix // page)
    w = None
    g = torch.Generator().manual_seed(1)
    rand = lambda *z: torch.randn(z, generator=g).to(dtype).cuda()  # noqa: E731
    tol = 2e-2 if dtype == BF else 1e-4

    def step():
        nonlocal w, now
        B.adacluster_cache_append(p, rand(3, Hkv, d), rand(3, Hkv, d), cu, now, table, cache)
        now = now + 1
        q = rand(3, Hq, d)
        o, lse = B.adacluster_prefix_attn(p, q, cu, cache, now, table, **groups)
        o2, lse2 = B.adacluster_block_attn(p, q, cu, cache=cache, seq_lens=now, page_table=table)
        assert float((o.float() - o2.float()).abs().max()) <= tol and float((lse - lse2).abs().max()) <= 1e-3
        w = B.adacluster_cache_weights(p, q, cu, lse, cache, now, table, weights=w, decay=1.0)
        return q, o, lse

    for _ in range(steps):
        step()
    # every step's rows weigh one in all
    assert float((w.double().sum(2) - steps * Hq // Hkv).abs().max()) <= 1e-2
    keep, recent = 61, 4
    new_table = torch.full_like(table, -1)
    new_table[:, :prefix // page] = table[:, :prefix // page]
    for b in range(3):
        for pg in range(prefix // page, x.max_pages):
            new_table[b, pg] = free.pop()
    cu_old = torch.tensor([0] + torch.cumsum(now.cpu(), 0).tolist(), dtype=torch.int32).cuda()
    p_all = replace(p, max_q=256)
    zero = torch.zeros_like(now)
    k_old, v_old = B.adacluster_cache_read(p_all, cache, cu_old, zero, table, rows=int(now.sum()))
    kept, lens_new, w_new = B.adacluster_cache_evict(p, cache, now, table, w, keep, recent, new_table)
    assert lens_new.tolist() == [keep] * 3
    cu_new = torch.arange(0, 4, dtype=torch.int32, device="cuda") * keep
    k_new, v_new = B.adacluster_cache_read(p_all, cache, cu_new, zero, new_table, rows=3 * keep)
    for b in range(3):
        assert kept[b, :, :prefix].tolist() == [list(range(prefix))] * Hkv
        for h in range(Hkv):
            stay = kept[b, h].long()
            assert torch.equal(k_new[b * keep:(b + 1) * keep, h], k_old[int(cu_old[b]) + stay, h])
            assert torch.equal(v_new[b * keep:(b + 1) * keep, h], v_old[int(cu_old[b]) + stay, h])
            assert torch.equal(w_new[b, h, :keep], w[b, h, stay]) and bool((w_new[b, h, keep:] == 0).all())
    table, now, w = new_table, lens_new, w_new
    for _ in range(3):
        step()
    sel, _ = B.adacluster_block_select(replace(p, topk=8), rand(3, Hq, d), cu, cache.boxes, seq_lens=now, page_table=table)
    assert bool((sel[..., 0] == 0).all())
