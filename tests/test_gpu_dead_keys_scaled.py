"""Clustered and dense attention over keys of -inf at soft-max scales above 1 / log2(e), where the lowest float divided by the scale
and scaled again rounds to minus infinity: whole tiles of such keys weigh nothing."""
import numpy as np
import pytest

from paper_2604_18348_amd import binding as B
from paper_2604_18348_amd import workloads as wl
from tests.test_gpu_attention import check, reference_with_dead_keys, to_dev, to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.88, 0.97, 1.3, 1.53, 2.72])
@pytest.mark.parametrize("dtype,d,H,N", [(B.BF16, 64, 1, 2500), (B.BF16, 128, 2, 2049),          # in pieces of the key list
                                         (B.BF16, 64, 30, 545), (B.BF16, 128, 9, 1025),          # whole lists
                                         (B.F32, 64, 2, 600), (B.F32, 128, 1, 33), (B.F32, 64, 70, 545)])
def test_tiles_of_dead_keys_at_any_scale(dtype, d, H, N, scale):
    rng = np.random.default_rng(31)
    make = lambda a: wl.round_bf16_f32(a) if dtype == B.BF16 else a  # noqa: E731
    # scores about as large as at the usual scale
    Q = make((rng.random((H, N, d)).astype(np.float32) + 0.1) / np.float32(scale * d ** 0.5))
    K, V = (make(rng.standard_normal((H, N, d)).astype(np.float32)) for _ in range(2))
    scale = float(np.float32(scale))
    for dead in (np.arange(N * 3 // 4, N), np.arange(min(N - 1, 161)), np.arange(N - 1), np.arange(1, N)):
        K2 = K.copy()
        K2[:, dead] = -np.inf
        p = B.Params(H=H, N=N, d=d, dtype=dtype, q_clusters=1, k_m0=1, k_m_min=1, k_max_clusters=1, softmax_scale=scale)
        O = to_np(B.adacluster_dense_attn(p, to_dev(Q, dtype), to_dev(K2, dtype), to_dev(V, dtype)))
        for h in (0, H - 1):
            check(O[h], reference_with_dead_keys(Q[h], K[h], V[h], dead, scale), dtype)
