"""Attention over shared prefixes of queries that lie in a tensor of more rows than the call can have queries (a buffer for the largest batch, rows of
sequences with more queries than max_q): against the definition in 64 bits, and rows that belong to no query left as they were."""
from dataclasses import replace

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests.test_gpu_blocks import BF, F, Batch
from tests.test_gpu_prefix import Shared

pytestmark = pytest.mark.gpu

LAYOUTS = [  # d, page, Hq, Hkv, lens, news, cu_group, prefix, max_q
    (64, 16, 4, 4, [1], [1], [0, 1], [1], 1),
    (128, 16, 8, 2, [333, 300, 290, 1, 40], [1, 1, 1, 1, 1], [0, 3, 5], [289, 1], 1),
    (128, 32, 12, 4, [700, 641, 641, 900, 650], [1, 1, 0, 1, 1], [0, 3, 3, 5], [640, 5, 641], 1),      # a group and a sequence without queries
    (64, 64, 6, 2, [500, 0, 450, 131], [1, 1, 1, 1], [1, 2, 4], [300, 130], 1),                       # a sequence outside, one without keys
    (64, 16, 15, 3, [200, 180, 170], [5, 3, 4], [0, 3], [167], 5),
    (64, 16, 8, 1, [500 + i for i in range(12)], [1] * 12, [0, 5, 12], [480, 333], 1),                # tiles of many rows
    (128, 16, 16, 4, [900 + 3 * i for i in range(40)], [1 + i % 4 for i in range(40)], [0, 17, 40], [890, 801], 4),
    (128, 16, 16, 4, [900 + 3 * i for i in range(40)], [1 + i % 7 for i in range(40)], [0, 17, 40], [890, 801], 3),      # more queries than max_q
    (64, 128, 6, 2, [700 - i for i in range(30)], [i % 5 for i in range(30)], [0, 20, 21, 30], [680, 600, 670], 2),
    (128, 32, 8, 2, [400, 380, 401], [60, 80, 33], [0, 3], [352], 50),                                # queries that the prefix cuts
    (64, 64, 12, 1, [1400 + i for i in range(12)], [1] * 12, [0, 12], [1399], 1),
]


@pytest.mark.parametrize("spare", [500, 70000])
@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_spare_rows(layout, dtype, bits, spare):
    d, page, Hq, Hkv, lens, news, cu_group, prefix, max_q = layout
    x = Batch(dtype, bits, d, page, Hq, Hkv, lens, news, 9, spare=spare)
    s = Shared(x, cu_group, prefix)
    p = replace(x.params(), max_q=max_q)
    q = x.q.cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0], Hq), 7.0, device="cuda")
    B.adacluster_prefix_attn(p, q, x.cu_q.cuda(), x.cache, **s.ints(), out=out, lse=lse)
    s.check(p, out, lse, max_q=max_q)
    mine = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for b, nq in enumerate(news):
        mine[int(x.cu_q[b]):int(x.cu_q[b]) + min(nq, max_q)] = True
    assert bool((out[~mine] == 7).all()) and bool((lse[~mine] == 7).all())
    if max(news) <= 1 and min(news) == 1:                        # rows counted either way are the same tiles: the same bits
        n = int(x.cu_q[-1])
        a, b = B.adacluster_prefix_attn(p, q[:n], x.cu_q.cuda(), x.cache, **s.ints())
        assert torch.equal(a, out[:n]) and torch.equal(b, lse[:n])


def test_rows_before_the_first_sequence():
    x = Batch(BF, 0, 64, 16, 8, 2, [300 + i for i in range(9)], [1 + i % 3 for i in range(9)], 4, spare=400)
    s = Shared(x, [0, 4, 9], [280, 290])
    q = torch.cat([torch.zeros_like(x.q[:333]), x.q]).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0], 8), 7.0, device="cuda")
    B.adacluster_prefix_attn(x.params(), q, x.cu_q.cuda() + 333, x.cache, **s.ints(), out=out, lse=lse)
    s.check(x.params(), out[333:], lse[333:])
    assert bool((out[:333] == 7).all()) and bool((lse[:333] == 7).all())


def test_wild_device_data():
    """Groups, lengths and rows are held to the buffers here too."""
    x = Batch(BF, 0, 64, 16, 4, 2, [160, 150, 140], [1, 1, 1], 4, spare=100)
    s = Shared(x, [0, 3], [96])
    ints = s.ints()
    for name, value in (("cu_group", [-5, 1 << 30]), ("cu_group", [3, 0]), ("prefix_lens", [1 << 30]), ("seq_lens", [1 << 30, -7, 50])):
        B.adacluster_prefix_attn(x.params(), x.q.cuda(), x.cu_q.cuda(), x.cache, **{**ints, name: torch.tensor(value, dtype=torch.int32).cuda()})
    for cu in ([0, 1 << 30, -3, 2], [9, 9, 9, 9], [3, 2, 1, 0]):
        B.adacluster_prefix_attn(x.params(), x.q.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), x.cache, **ints)
    torch.cuda.synchronize()
