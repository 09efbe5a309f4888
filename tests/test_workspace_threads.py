"""The binding's cached workspace is a host thread's own: calls of two threads at once must not share scratch (no GPU needed)."""
import os
import threading

from paper_2604_18348_amd import binding as B


def test_threads_have_workspaces_of_their_own():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_18348_amd import build
        build.build()
    p = B.Params(H=2, N=2600, d=64, dtype=B.BF16, q_clusters=9, q_iters=3, k_iters=3, k_m0=16, k_m_min=4, k_max_clusters=64,
                 min_unassigned_frac=0.03, topk=5)
    got = []

    def work():
        got.append((B.workspace(p, "cpu"), B.workspace(p, "cpu")))

    for _ in range(2):                                           # (one after the other; what the first one got is still held)
        t = threading.Thread(target=work)
        t.start()
        t.join()
    (a, again), (b, _) = got
    assert a.data_ptr() == again.data_ptr()                      # kept from call to call
    lo, hi = sorted((a, b), key=lambda t: t.data_ptr())
    assert lo.data_ptr() + lo.numel() <= hi.data_ptr()
