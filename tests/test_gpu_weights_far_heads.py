"""Weights of cached keys from queries whose many heads lie far apart, against the definition in 64 bits (bounds: tests/test_gpu_keep.py): offsets up to
the 2^32 bytes that the kernel for many rows holds, and past them."""
import math

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests.test_gpu_blocks import BF, Batch, _within
from tests.test_gpu_keep import _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("G,head", [(160, 1 << 22), (160, 13500000), (160, 13600000), (160, (1 << 24) - 64), (131, (1 << 24) - 64), (129, (1 << 24) - 64)])
def test_many_heads_far_apart(G, head, bits):
    head -= head % 8
    x = Batch(BF, bits, 64, 16, G, 1, [90], [4], 6)
    p, q, cu = x.params(), x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    want, tol = _weights(x, 0, lse.cpu(), 1 / math.sqrt(64), 1, None)
    far = torch.zeros((G - 1) * head + q.shape[0] * 64, dtype=BF, device="cuda")
    view = far.as_strided(q.shape, (64, head, 1))
    view.copy_(q)
    got = B.adacluster_cache_weights(p, view, cu, lse, x.cache, **x.where())
    _within(got[0, :, :90], want, tol, "weights, %d heads %d apart" % (G, head))


@pytest.mark.parametrize("bits", [0, 4])
def test_tokens_far_apart_of_many_heads(bits):
    G, token = 150, (1 << 24) - 64
    x = Batch(BF, bits, 64, 16, G, 1, [90], [4], 6)
    p, q, cu = x.params(), x.q.cuda(), x.cu_q.cuda()
    _, lse = B.adacluster_block_attn(p, q, cu, cache=x.cache, **x.where())
    want, tol = _weights(x, 0, lse.cpu(), 1 / math.sqrt(64), 1, None)
    far = torch.zeros(q.shape[0] * token, dtype=BF, device="cuda")
    view = far.as_strided(q.shape, (token, 64, 1))
    view.copy_(q)
    got = B.adacluster_cache_weights(p, view, cu, lse, x.cache, **x.where())
    _within(got[0, :, :90], want, tol, "weights, tokens %d apart" % token)
