"""The binding's cached workspace belongs to a stream, and a captured graph has one of its own: on the host, with streams in name only (no GPU needed;
tests/test_gpu_workspace_streams.py has the calls)."""
import os

import pytest
import torch

from paper_2604_18348_amd import binding as B

P = B.Params(H=2, N=2600, d=64, dtype=B.BF16, q_clusters=9, q_iters=3, k_iters=3, k_m0=16, k_m_min=4, k_max_clusters=64,
             min_unassigned_frac=0.03, topk=5)


@pytest.fixture
def on(monkeypatch):
    """Makes a stream the current one: on(stream, captured)"""
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    state, empty = dict(stream=0, captured=False), torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, **{**kw, "device": "cpu"}))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["captured"])
    monkeypatch.setattr(B, "_raw_stream", lambda i: state["stream"])
    return lambda stream, captured=False: state.update(stream=stream, captured=captured)


def test_streams(on):
    got = []
    for s in (0, 7, 9):
        on(s)
        got.append(B.workspace(P, "cuda"))
    assert len({t.data_ptr() for t in got}) == 3
    for s, t in zip((0, 7, 9), got):
        on(s)
        assert B.workspace(P, "cuda:0").data_ptr() == B.workspace(P, "cuda").data_ptr() == t.data_ptr()


def test_graphs(on):
    on(7)
    kept = B.workspace(P, "cuda")
    on(7, True)
    first, second = B.workspace(P, "cuda"), B.workspace(P, "cuda")
    assert len({t.data_ptr() for t in (kept, first, second)}) == 3
    on(7)
    assert B.workspace(P, "cuda").data_ptr() == kept.data_ptr()
