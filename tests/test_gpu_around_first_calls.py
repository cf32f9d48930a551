"""The norm, the E4M3 rows' product, the balance loss and the orthogonalised update from where nothing has run yet: inside a capture, on a host
thread that has made no CUDA call, and on several threads at once."""
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2602_06183_b200 import binding as b

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, U8 = torch.bfloat16, torch.uint8


def _normal(*shape):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(sum(shape)), device="cuda")


def norm(T, s=None):
    D = 520
    X, R, dY, G = _normal(T, D).to(BF), _normal(D, T).T.contiguous().to(BF), _normal(1, T, D)[0].to(BF), _normal(D).to(BF)
    S, Y, dX, dg = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(G)
    q, sc, rstd = torch.zeros((T, D), dtype=U8, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    ws = torch.zeros(b.sf_rmsnorm_bwd_workspace_size(T, D), dtype=U8, device="cuda")

    def run():
        b.sf_rmsnorm_fwd(X, G, 1e-6, residual=R, sum=S, Y=Y, codes=q, scales=sc, rstd=rstd, stream=s)
        b.sf_rmsnorm_bwd(dY, S, G, rstd, dX=dX, dgamma=dg, workspace=ws, stream=s)
    return run, [S, Y, q, sc, rstd, dX, dg]


def rows(M, s=None):
    N, K = 264, 528
    A, B = (_normal(n, K).to(torch.float8_e4m3fn).view(U8) for n in (M, N))
    sc, C, ws = _normal(M).abs(), torch.zeros((M, N), dtype=BF, device="cuda"), torch.zeros(256, dtype=U8, device="cuda")
    return lambda: b.sf_gemm_fp8_rows(A, sc, B, 0.5, C_out=C, workspace=ws, stream=s), [C]


def balance(T, s=None):
    D, E = 136, 6
    X, m = _normal(T, D).to(BF), (_normal(E, D) * 0.1).to(BF)
    L = X.float() @ m.float().T
    ex = L.argmax(1).int()
    loss, n, dX, dm = torch.zeros(3, device="cuda"), torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros_like(X), torch.zeros_like(m)
    ws = torch.zeros(b.sf_router_balance_workspace_size(T, D, E), dtype=U8, device="cuda")

    def run():
        b.sf_router_balance_fwd(L, ex, 0.5, 0.1, loss=loss, counts=n, workspace=ws, stream=s)
        b.sf_router_balance_bwd(L, ex, n, 0.5, 0.1, X, m, dX=dX, dmeans=dm, workspace=ws, stream=s)
    return run, [loss, n, dX, dm]


def update(m, s=None):
    G = _normal(m, 2 * m).to(BF)
    O, ws = torch.zeros_like(G), torch.zeros(b.sf_orthogonalize_workspace_size(m, 2 * m), dtype=U8, device="cuda")
    return lambda: b.sf_orthogonalize(G, out=O, workspace=ws, stream=s), [O]


CASES = [(norm, 5), (norm, 300), (rows, 3), (rows, 100), (rows, 200), (balance, 4), (balance, 3000), (update, 24), (update, 100), (update, 200), (update, 1100)]
CAPTURE = """
import sys, torch
sys.path.insert(0, "tests")
import test_gpu_around_first_calls as t
for make, n in t.CASES:
    run, out = make(n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in out]
    for x in out: x.zero_()
    run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(out, got)), (make.__name__, n)
"""
THREADS = """
import sys, threading, torch
sys.path.insert(0, "tests")
import test_gpu_around_first_calls as t
for make, n in t.CASES:
    jobs, gate, failed = [make(n, torch.cuda.Stream()) for _ in range(4)], threading.Barrier(4), []
    torch.cuda.synchronize()
    def go(run):
        gate.wait()
        try:
            run()
        except Exception as e:
            failed.append(e)
    threads = [threading.Thread(target=go, args=(run,)) for run, _ in jobs]
    for x in threads: x.start()
    for x in threads: x.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for _, out in jobs:
        assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(out, jobs[0][1])), (make.__name__, n)
"""


@pytest.mark.parametrize("code", [CAPTURE, THREADS], ids=["captured", "threads"])
def test_first_calls(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]


@pytest.mark.parametrize("make,n", CASES)
def test_first_cuda_call_of_a_thread(make, n):
    s, failed = torch.cuda.Stream(), []
    run, out = make(n, s)
    torch.cuda.synchronize()
    run()
    s.synchronize()
    want = [t.clone() for t in out]
    for t in out:
        t.zero_()
    torch.cuda.synchronize()

    def go():
        try:
            run()
        except Exception as e:
            failed.append(e)
    thread = threading.Thread(target=go)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert not failed, failed
    assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(out, want))
