"""Weights of cached keys by the queries of a sequence inside a tensor of very many rows and heads (strides of 0: its rows are one)."""
import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests.test_gpu_blocks import BF, Batch

pytestmark = pytest.mark.gpu


def test_more_rows_and_heads_than_a_launch_has_lanes():
    """2^30 rows and heads, of which a sequence has 40 x 64: what the same 40 rows alone give."""
    x = Batch(BF, 0, 64, 16, 64, 1, [100], [40], 6)
    p, cu = x.params(), x.cu_q.cuda()
    q = x.q[:1, :1].cuda()
    few = q.expand(40, 64, 64)
    _, lse = B.adacluster_block_attn(p, few, cu, cache=x.cache, out=torch.empty((40, 64, 64), dtype=BF, device="cuda"), **x.where())
    want = B.adacluster_cache_weights(p, few, cu, lse, x.cache, **x.where())
    rows = (1 << 24) + 64
    many = torch.empty((rows, 64), device="cuda")
    many[:40] = lse
    got = B.adacluster_cache_weights(p, q.expand(rows, 64, 64), cu, many, x.cache, **x.where())
    assert torch.equal(got, want) and float(got.sum()) > 1
