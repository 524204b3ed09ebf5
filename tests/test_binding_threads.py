"""Workspaces that the binding keeps: one per thread, since the launches of two threads may take turns on one stream, and none for a call
that is captured, which gets one of its own."""
import sys
import threading

import numpy as np
import pytest
import torch

from paper_2311_00368_b200 import build as b2sp_build


@pytest.fixture(scope="module")
def b():
    b2sp_build.build()
    from paper_2311_00368_b200 import binding
    return binding


def _in_threads(n, fn):
    """fn(i) in n threads at once; their results."""
    out, errors, gate = [None] * n, [], threading.Barrier(n)

    def run(i):
        try:
            gate.wait(60)
            out[i] = fn(i)
            gate.wait(60)   # (all live to the end: nothing is handed back before the others have theirs)
        except BaseException as e:  # noqa: BLE001
            errors.append(e)
            gate.abort()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(n)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]
    return out


def test_each_thread_has_a_workspace_of_its_own(b, monkeypatch):
    monkeypatch.setattr(b, "_capturing", lambda: False)
    monkeypatch.setattr(b, "_raw_stream", lambda i: 0)
    cpu = torch.device("cpu")
    for get in (lambda: b._scratch(5000, cpu, None, 0), lambda: b._workspace(b.OP_SPMM, 64, 64, 0, 64, 100, cpu, None)[0]):
        def twice(i):
            a = get()
            assert get().data_ptr() == a.data_ptr()
            return a
        kept = _in_threads(4, twice)
        assert len({t.data_ptr() for t in kept}) == 4


def test_a_captured_call_has_a_workspace_of_its_own(b, monkeypatch):
    monkeypatch.setattr(b, "_raw_stream", lambda i: 0)
    cpu = torch.device("cpu")
    for get in (lambda: b._scratch(5000, cpu, None, 0), lambda: b._workspace(b.OP_SPMM, 64, 64, 0, 64, 100, cpu, None)[0]):
        monkeypatch.setattr(b, "_capturing", lambda: False)
        kept = get()
        monkeypatch.setattr(b, "_capturing", lambda: True)
        one, other = get(), get()
        assert len({t.data_ptr() for t in (kept, one, other)}) == 3
        monkeypatch.setattr(b, "_capturing", lambda: False)
        assert get().data_ptr() == kept.data_ptr()


@pytest.mark.gpu
def test_two_graphs_of_a_matrix_product(b):
    """Captured on one stream, replayed at once on two: neither disturbs the other."""
    from paper_2311_00368_b200 import workloads as W
    calls, want, graphs, outs = [], [], [], []
    for i in range(2):
        p = W.small_random(1030 + i, 2000, 2000, 0.2, 64, 64)
        rp, ci, A, B, D = (torch.from_numpy(x).cuda() for x in (p.row_ptr, p.col_idx, p.A, p.B, p.D))
        calls.append(lambda rp=rp, ci=ci, A=A, B=B, D=D: b.fusedmm(rp, ci, None, A, B, D, algo=b.ALGO_TILE))
        want.append(calls[-1]())
    torch.cuda.synchronize()
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c())
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for x, y in zip(outs, want):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, d", [(torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 100), (torch.bfloat16, 83)])
@pytest.mark.parametrize("algo", [1, 3])
def test_two_threads_on_one_stream(b, algo, dtype, d):
    """Calls of several kernels (rows in parts, cut blocks, shares, planes, products in memory) from two threads on the default stream give
    what they give alone, to the bit."""
    from tests.test_gpu_attention import Problem
    ps = [Problem(1000 + i, H=2, M=140 + 60 * i, K=2600, d=d, dtype=dtype) for i in range(2)]
    plans = [p.plan() for p in ps]

    def call(i):
        o, lse = ps[i].forward(algo, plans[i])
        return (o, lse, *ps[i].backward(o, lse, plans[i], algo))
    want = [call(i) for i in range(2)]
    torch.cuda.synchronize()
    _race(lambda i: [call(i) for _ in range(30)], want)


@pytest.mark.gpu
def test_two_threads_over_caches(b):
    from tests.test_gpu_kv4 import Served
    ss = [Served(1010 + i, [3000, 7, 900], 8, 2, 128, 3000) for i in range(2)]
    want = [s.run() for s in ss]
    _race(lambda i: [ss[i].run() for _ in range(50)], want)


@pytest.mark.gpu
def test_two_threads_of_matrix_products(b):
    from paper_2311_00368_b200 import workloads as W
    calls = []
    for i in range(2):
        p = W.small_random(1020 + i, 600 + 100 * i, 700, 0.2, 64, 64)
        rp, ci, A, B, D = (torch.from_numpy(x).cuda() for x in (p.row_ptr, p.col_idx, p.A, p.B, p.D))
        calls.append(lambda rp=rp, ci=ci, A=A, B=B, D=D: tuple(b.fusedmm(rp, ci, None, A, B, D, algo=a) for a in (b.ALGO_ROW, b.ALGO_TILE)))
    want = [c() for c in calls]
    _race(lambda i: [calls[i]() for _ in range(50)], want)


def _race(fn, want):
    """fn(i) in a thread for each i, on the default stream, with turns as short as they get: every result is want[i], to the bit."""
    was = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        got = _in_threads(len(want), fn)
    finally:
        sys.setswitchinterval(was)
    torch.cuda.synchronize()
    for results, ref in zip(got, want):
        for one in results:
            for x, y in zip(one, ref):
                assert np.array_equal(torch.nan_to_num(x).float().cpu().numpy(), torch.nan_to_num(y).float().cpu().numpy())
