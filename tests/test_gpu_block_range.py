"""Attention over pages with values as large as the interface allows, and scores that rise as far as they can before weights are scaled down."""
import math

import pytest
import torch

from paper_2604_18348_amd import binding as B
from tests import block_reference as ref
from tests.test_gpu_blocks import BF, F, Batch, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bits", [(BF, 0), (F, 0), (BF, 4), (F, 4)])
@pytest.mark.parametrize("Hq,Hkv,n,nq", [(4, 2, 1200, 1), (2, 1, 900, 40), (64, 1, 700, 256)])
def test_the_largest_values(Hq, Hkv, n, nq, dtype, bits):
    """Keys 0 to 127 (the first turn of every wave) have score 0, the others 15.9 log 2: no weight moves the reference, and their sum is
    that of nearly 2^16 a key."""
    x = Batch(dtype, bits, 64, 16, Hq, Hkv, [n], [nq], 71, spare=0)
    g = torch.Generator().manual_seed(1)
    most = 2.0 ** (108 if bits else 112) / n
    x.q = torch.ones_like(x.q)
    k, v = torch.zeros((n, Hkv, 64)), (torch.rand((n, Hkv, 64), generator=g) * 0.98 + 0.01) * most * torch.sign(torch.randn((1, Hkv, 64), generator=g))
    k[128:] = 15.9 * math.log(2) / 64
    x.k, x.v = k.to(dtype), v.to(dtype)
    p = x.params(causal=0, softmax_scale=1.0)
    cache = B.alloc_cache(p, x.max_pages)
    table = torch.arange(x.max_pages, dtype=torch.int32, device="cuda").view(1, -1)
    lens, old, cu = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in ([n], [0], [0, n]))
    fill = B.BlockParams(**{**p.__dict__, "max_q": n})
    B.adacluster_cache_append(fill, x.k.cuda(), x.v.cuda(), cu, old, table, cache)
    o, lse = B.adacluster_block_attn(p, x.q.cuda(), x.cu_q.cuda(), cache=cache, seq_lens=lens, page_table=table)
    kr, vr, ka, va = x.k, x.v, None, None
    if bits:
        kr, vr = (ref.dequantise(*ref.quantise(t)) for t in (x.k, x.v))
        ka, va = ((143 * m[..., 0] + m[..., 1].abs()).repeat_interleave(64, -1) for m in (ref.quantise(t)[1].double() for t in (x.k, x.v)))
    r = ref.attend(x.q, kr, vr, ref.sees(None, n, nq, Hkv, 16, 1, 0), 1.0, dtype, ka, va)
    assert bool(o.isfinite().all())
    _within(o, r["o"], r["o_tol"], "o")
    _within(lse, r["lse"], r["lse_tol"], "lse")
