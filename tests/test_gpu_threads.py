"""Calls from host threads of their own: a thread that has made no CUDA call yet, and several first calls at once."""
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2602_06183_b200 import binding as b

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF = torch.bfloat16


def _normal(*shape):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(sum(shape)), device="cuda").to(BF)


def _gated(T, s):
    D, F = 136, 264
    t = [_normal(T, D), _normal(T, D) * 0.5, _normal(F, D) * 0.1, _normal(F, D) * 0.2, _normal(D, F) * 0.1]
    out = [torch.zeros_like(t[i]) for i in (1, 1, 2, 3, 4)]
    d = b.make_gated_desc(T, D, F)
    ctx, ws = b.alloc_gated_ffn_buffers(d)

    def run():
        b.sf_gated_ffn_fwd(d, *t[1:], out[0], ctx, ws, stream=s)
        b.sf_gated_ffn_bwd(d, *t, ctx, *out[1:], ws, stream=s)
    return run, out


def _fp4(M, s):
    N, K = 264, 512
    x, w = b.sf_fp4_quantize(_normal(M, K), b.SF_FP4_NV, 2.0), b.sf_fp4_quantize(_normal(N, K), b.SF_FP4_NV, 2.0)
    C, ws = torch.zeros((M, N), dtype=BF, device="cuda"), torch.zeros(256, dtype=torch.uint8, device="cuda")
    return lambda: b.sf_gemm_fp4(*x, *w, b.SF_FP4_NV, 0.25, C_out=C, workspace=ws, stream=s), [C]


def _quantize(M, s):
    x = _normal(M, 512)
    q = tuple(torch.zeros_like(t) for t in b.sf_fp4_quantize(x, b.SF_FP4_MX, 2.0))
    y = torch.zeros_like(x)

    def run():
        b.sf_fp4_quantize(x, b.SF_FP4_MX, 2.0, out=q, stream=s)
        b.sf_fp4_dequantize(*q, b.SF_FP4_MX, 0.5, out=y, stream=s)
    return run, [y, *q]


def _sparse(T, s):
    D, F = 256, 512
    d = b.make_desc(T, D, F, 64, 8)
    t = [_normal(T, D), _normal(T, D) * 0.5, _normal(F, D) * 0.1, _normal(F, D) * 0.2]
    ctx, ws = b.alloc_ffn_buffers(d)
    out = [torch.zeros_like(t[i]) for i in (1, 1, 2, 3)]

    def run():
        b.sf_sparse_ffn_fwd(d, *t[1:], out[0], ctx, ws, stream=s)
        b.sf_sparse_ffn_bwd(d, *t, ctx, *out[1:], ws, stream=s)
    return run, out


def _fp8(M, s):
    a, w = b.sf_fp8_quantize(_normal(M, 512), 2.0), b.sf_fp8_quantize(_normal(256, 512), 2.0)
    C, ws = torch.zeros((M, 256), dtype=BF, device="cuda"), torch.zeros(b.sf_gemm_fp8_workspace_size(M, 512), dtype=torch.uint8, device="cuda")
    return lambda: b.sf_gemm_fp8_dense(a, w, 0.25, C_out=C, workspace=ws, stream=s), [C]


@pytest.mark.parametrize("make,T", [(_gated, 5), (_gated, 40), (_gated, 300), (_fp4, 3), (_fp4, 300), (_quantize, 70), (_sparse, 256), (_fp8, 256)])
def test_first_cuda_call_of_a_thread(make, T):
    s, failed = torch.cuda.Stream(), []
    run, out = make(T, s)
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


CODE = """
import sys, threading, torch
sys.path.insert(0, "tests")
import test_gpu_threads as t
for make, T in ((t._gated, 5), (t._gated, 40), (t._gated, 200), (t._fp4, 3), (t._fp4, 300), (t._sparse, 256)):
    blocks, gate, failed = [make(T, torch.cuda.Stream()) for _ in range(6)], threading.Barrier(6), []
    torch.cuda.synchronize()
    def go(run):
        gate.wait()
        try:
            run()
        except Exception as e:
            failed.append(e)
    threads = [threading.Thread(target=go, args=(run,)) for run, _ in blocks]
    for x in threads: x.start()
    for x in threads: x.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for _, out in blocks:
        assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(out, blocks[0][1])), (make.__name__, T)
"""


def test_first_calls_of_several_threads_at_once():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
