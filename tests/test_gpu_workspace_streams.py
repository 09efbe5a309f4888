"""The binding's cached workspace belongs to a host thread and a stream, and a captured graph has one of its own."""
import dataclasses
import threading

import pytest
import torch

from paper_2604_18348_amd import binding as B
from paper_2604_18348_amd import workloads as wl
from tests.helpers import to_dev

pytestmark = pytest.mark.gpu

P = B.Params(H=2, N=2600, d=64, dtype=B.BF16, q_clusters=9, q_iters=3, k_iters=3, k_m0=16, k_m_min=4, k_max_clusters=64,
             min_unassigned_frac=0.03, topk=5)


def _apart(*ts):
    at = sorted((t.data_ptr(), t.numel()) for t in ts)
    return all(a + n <= b for (a, n), (b, _) in zip(at, at[1:]))


def test_streams_of_one_thread_have_workspaces_of_their_own():
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [B.workspace(P)]
    for s in side:
        with torch.cuda.stream(s):
            got.append(B.workspace(P, "cuda:0"))
    assert _apart(*got)
    for s, want in zip((torch.cuda.default_stream(), *side), got):      # kept from call to call, whatever the device is called
        with torch.cuda.stream(s):
            for dev in ("cuda", "cuda:0", torch.device("cuda", 0)):
                assert B.workspace(P, dev).data_ptr() == want.data_ptr()


def test_two_streams_of_one_thread_at_once():
    """Calls without `ws`, enqueued on two streams in turn (a warm start waits for nothing): each gives what it gives alone."""
    cases = []
    for seed in (41, 42):
        Q, K, V = (to_dev(x, B.BF16) for x in wl.make_small(seed, P.N, P.d, 10, dtype="bf16", H=P.H))
        outs = B.alloc_outputs(P, "cuda")
        B.adacluster_attn(P, Q, K, V, outs=outs)
        cases.append((Q, K, V, outs))
    warm = dataclasses.replace(P, q_init_mode=1, k_init_mode=1, q_iters=2, k_iters=2)
    start = [{k: t.clone() for k, t in c[3].items() if t is not None} for c in cases]

    def state():
        return [{**c[3], **{k: t.clone() for k, t in s.items()}} for c, s in zip(cases, start)]

    alone = [[B.adacluster_attn(warm, *c[:3], outs=o) for _ in range(4)] for c, o in zip(cases, state())]
    outs = state()
    torch.cuda.synchronize()
    side, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(4):
        for i, s in enumerate(side):
            with torch.cuda.stream(s):
                got[i].append(B.adacluster_attn(warm, *cases[i][:3], outs=outs[i]))
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_graph_outlives_the_thread_that_captured_it():
    """Captured without `ws`, after a warm-up, in a thread that ends: replays give what eager calls give, whatever has been allocated since."""
    Q, K, V = (to_dev(x, B.BF16) for x in wl.make_small(43, P.N, P.d, 10, dtype="bf16", H=P.H))
    outs, O = B.alloc_outputs(P, "cuda"), torch.empty_like(Q)
    B.adacluster_attn(P, Q, K, V, outs=outs, out=O)
    warm = dataclasses.replace(P, q_init_mode=1, k_init_mode=1, q_iters=2, k_iters=2)
    start = {k: t.clone() for k, t in outs.items() if t is not None}

    def restore():
        for k, t in start.items():
            outs[k].copy_(t)
        torch.cuda.synchronize()

    eager = []
    for _ in range(3):
        eager.append(B.adacluster_attn(warm, Q, K, V, outs=outs).clone())
    held, errs = [], []

    def work():
        try:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            before = B.workspace(warm)
            with torch.cuda.graph(g):
                during = B.workspace(warm)
                B.adacluster_attn(warm, Q, K, V, outs=outs, out=O)
            assert _apart(before, during) and B.workspace(warm).data_ptr() == before.data_ptr()
            held.append(g)
        except Exception as e:      # surfaced in the main thread
            errs.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    assert not errs, errs
    restore()
    for r in range(3):
        junk = [torch.full((B.adacluster_workspace_bytes(P) // 4 + 64,), 0x7F7F7F7F, dtype=torch.int32, device="cuda") for _ in range(6)]
        torch.cuda.synchronize()
        held[0].replay()
        torch.cuda.synchronize()
        assert torch.equal(O, eager[r]), r
        assert all(bool((j == 0x7F7F7F7F).all()) for j in junk)
        B.workspace(dataclasses.replace(P, N=900))              # one of another size: nothing that the graph uses goes with the old one
