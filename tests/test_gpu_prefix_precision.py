"""How exact attention over shared prefixes is in bfloat16: as in adacluster_block_attn of one token, weights lose 2^-16 before they meet the values, so a
result is off by its own rounding and by what sums in 32 bits lose, however many rows share the keys, and over 4-bit caches too.  (Blocks of 128
rows of a sequence, chunks of a prompt, have weights that are rounded once, as adacluster_block_attn does; tests/test_gpu_prefix.py bounds them.)

Bound: that of tests/block_reference.py for sums and scores in fp32 (no rounding of weights), 2^-16 of the sum of weights times |v| (half a step of
bfloat16, 2^-8, of what half a step has left), and half a step of the result."""
import math

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within
from tests.test_gpu_prefix import LAYOUTS, WIDE, Shared

pytestmark = pytest.mark.gpu


def rows_of_a_block(layout):
    G = layout[2] // layout[3]
    return G * min(max(1, 128 // G), max(1, max(layout[5])))


STEPS = [x for x in LAYOUTS + WIDE if rows_of_a_block(x) < 128]


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("layout", STEPS)
def test_results_are_rounded_once(layout, bits):
    d, page, Hq, Hkv, lens, news, cu_group, prefix = layout
    x = Batch(BF, bits, d, page, Hq, Hkv, lens, news, 9)
    s = Shared(x, cu_group, prefix)
    p = x.params()
    o, _ = B.adacluster_prefix_attn(p, x.q.cuda(), x.cu_q.cuda(), x.cache, **s.ints())
    for b in range(x.B):
        n, nq = x.lens[b], x.news[b]
        k, v, ka, va = s.keys(b)
        see = (torch.arange(n) <= n - nq + torch.arange(nq)[:, None])[:, None].expand(-1, Hkv, -1)
        q, scale = x.seq(x.q, b), 1 / math.sqrt(d)
        r = ref.attend(q, k, v, see, scale, F, ka, va)
        whole = ref.attend(q, k, v.double().abs() if va is None else va, see, scale, F, ka, va)["o"]
        tol = r["o_tol"] + 1.01 * (2.0 ** -16 * whole + ref.half(BF) * r["o"].abs())
        at = slice(int(x.cu_q[b]), int(x.cu_q[b + 1]))
        _within(o[at], r["o"], tol, "o of sequence %d" % b)


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("layout", [x for x in (LAYOUTS[2], LAYOUTS[4], LAYOUTS[5], *WIDE[:6], WIDE[7], WIDE[8]) if x in STEPS])
def test_results_are_the_rounded_definition_but_for_few(layout, bits):
    """What the bound above says little about over 4 bits (it counts codes as 128 + code).  A result that is off by e before it is rounded to steps of u
    lands on another one than the definition does once in u / e times, a step away: the squares of the differences are e u in the mean.  Sums of some
    hundred terms in fp32 are off by 2^-14 of a result or less, a step is 2^-8 to 2^-7 of it: 2^-11 relative to all results in the mean of squares, for
    which twice that is allowed.  (Weights rounded once leave 2^-8.7.)"""
    d, page, Hq, Hkv, lens, news, cu_group, prefix = layout
    x = Batch(BF, bits, d, page, Hq, Hkv, lens, news, 9)
    s = Shared(x, cu_group, prefix)
    o, _ = B.adacluster_prefix_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), x.cache, **s.ints())
    off = whole = 0.0
    for b in range(x.B):
        n, nq = x.lens[b], x.news[b]
        k, v, ka, va = s.keys(b)
        see = (torch.arange(n) <= n - nq + torch.arange(nq)[:, None])[:, None].expand(-1, Hkv, -1)
        want = ref.attend(x.seq(x.q, b), k, v, see, 1 / math.sqrt(d), F, ka, va)["o"].to(BF).double()
        off += float((o[int(x.cu_q[b]):int(x.cu_q[b + 1])].double().cpu() - want).square().sum())
        whole += float(want.square().sum())
    assert math.sqrt(off / whole) <= 2.0 ** -10
