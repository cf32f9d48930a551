"""What the norm, the E4M3 rows' product, the balance loss and the orthogonalised update refuse, on the host: nothing is launched (no GPU
needed, the pointers are fake)."""
import ctypes as C

import pytest
import torch

from paper_2602_06183_b200 import binding, build
from paper_2602_06183_b200.binding import (SF_ERR_ALIGN, SF_ERR_NULL, SF_ERR_SHAPE, SF_ERR_UNSUPPORTED, SF_ERR_WORKSPACE, SF_OK)

ODD, NONE = C.c_void_p(0x10008), None
AT = [C.c_void_p((i + 1) << 36) for i in range(12)]           # far from one another


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_norm(lib):
    T, D = 5, 64
    def fwd(X=AT[0], ldx=D, R=AT[1], g=AT[2], T=T, D=D, eps=1e-6, S=AT[3], Y=AT[4], q=AT[5], s=AT[6], r=AT[7]):
        return lib.sf_rmsnorm_fwd(X, ldx, R, g, T, D, eps, S, Y, q, s, 1.0, r, None)
    assert fwd(T=-1) == fwd(D=0) == fwd(D=60) == fwd(D=32776) == fwd(T=1 << 29) == SF_ERR_SHAPE
    assert fwd(X=NONE) == fwd(g=NONE) == fwd(Y=NONE, q=NONE, s=NONE) == fwd(q=NONE) == SF_ERR_NULL
    assert fwd(ldx=56) == fwd(ldx=68) == fwd(X=ODD) == fwd(R=ODD) == fwd(S=ODD) == fwd(Y=ODD) == fwd(q=ODD) == fwd(s=ODD) == fwd(r=ODD) == SF_ERR_ALIGN
    assert fwd(eps=-1e-6) == fwd(eps=float("nan")) == SF_ERR_UNSUPPORTED
    assert fwd(T=0, X=NONE, g=NONE) == SF_OK
    # shared bytes: the sum may be X (contiguous) or the residual, nothing else may meet anything
    assert fwd(Y=AT[0]) == fwd(Y=AT[1]) == fwd(S=AT[2]) == fwd(q=AT[4]) == fwd(S=AT[4]) == fwd(r=AT[6]) == SF_ERR_UNSUPPORTED
    assert fwd(S=AT[0], ldx=72) == fwd(S=C.c_void_p((1 << 36) + 16)) == fwd(S=AT[1], Y=AT[1]) == SF_ERR_UNSUPPORTED
    n = C.c_size_t()
    assert lib.sf_rmsnorm_bwd_workspace_size(T, D, NONE) == SF_ERR_NULL and lib.sf_rmsnorm_bwd_workspace_size(T, 63, C.byref(n)) == SF_ERR_SHAPE
    need = binding.sf_rmsnorm_bwd_workspace_size(T, D)
    def bwd(dY=AT[0], S=AT[1], g=AT[2], r=AT[3], dS=AT[4], T=T, D=D, dX=AT[5], dg=AT[6], w=AT[7], n=need):
        return lib.sf_rmsnorm_bwd(dY, S, g, r, dS, T, D, dX, dg, w, n, None)
    assert bwd(D=12) == SF_ERR_SHAPE
    assert bwd(dY=NONE) == bwd(S=NONE) == bwd(g=NONE) == bwd(r=NONE) == bwd(w=NONE) == SF_ERR_NULL
    assert bwd(dX=ODD) == bwd(dg=ODD) == bwd(dS=ODD) == bwd(w=ODD) == SF_ERR_ALIGN
    assert bwd(n=need - 1) == SF_ERR_WORKSPACE
    assert bwd(dX=AT[1]) == bwd(dg=AT[2]) == bwd(w=AT[0]) == bwd(dX=C.c_void_p((1 << 36) + 16)) == bwd(dg=AT[5]) == bwd(w=AT[4]) == SF_ERR_UNSUPPORTED
    assert bwd(dX=NONE, dg=NONE, dY=NONE) == SF_OK


def test_fp8_rows(lib):
    M, N, K = 5, 64, 48
    def run(A=AT[0], s=AT[1], B=AT[2], c=AT[3], M=M, N=N, K=K, w=AT[4], n=256):
        return lib.sf_gemm_fp8_rows(A, s, B, c, M, N, K, 1.0, w, n, None)
    assert run(M=-1) == run(N=60) == run(K=40) == run(K=0) == run(M=1 << 29) == SF_ERR_SHAPE
    assert run(A=NONE) == run(s=NONE) == run(B=NONE) == run(c=NONE) == run(w=NONE) == SF_ERR_NULL
    assert run(A=ODD) == run(s=ODD) == run(B=ODD) == run(c=ODD) == run(w=ODD) == SF_ERR_ALIGN
    assert run(n=255) == SF_ERR_WORKSPACE
    assert run(c=AT[0]) == run(c=AT[1]) == run(c=AT[2]) == run(c=AT[4]) == run(w=AT[1]) == SF_ERR_UNSUPPORTED
    assert run(M=0, A=NONE) == run(N=0, B=NONE) == SF_OK


def test_balance(lib):
    T, D, E = 40, 64, 5
    need = binding.sf_router_balance_workspace_size(T, D, E)
    def fwd(l=AT[0], ex=AT[1], T=T, E=E, loss=AT[2], n=AT[3], w=AT[4], wb=need):
        return lib.sf_router_balance_fwd(l, ex, T, E, 1.0, 0.0, loss, n, w, wb, None)
    assert fwd(T=-1) == fwd(E=0) == fwd(E=17) == SF_ERR_SHAPE
    assert fwd(l=NONE) == fwd(ex=NONE) == fwd(loss=NONE) == fwd(n=NONE) == fwd(w=NONE) == SF_ERR_NULL
    assert fwd(l=ODD) == fwd(ex=ODD) == fwd(loss=ODD) == fwd(n=ODD) == fwd(w=ODD) == SF_ERR_ALIGN
    assert fwd(wb=300) == SF_ERR_WORKSPACE
    assert fwd(loss=AT[0]) == fwd(n=AT[1]) == fwd(w=AT[0]) == fwd(loss=AT[3]) == SF_ERR_UNSUPPORTED
    def bwd(l=AT[0], ex=AT[1], n=AT[2], g=AT[3], X=AT[4], m=AT[5], T=T, D=D, E=E, d=AT[6], dX=AT[7], dm=AT[8], w=AT[9], wb=need):
        return lib.sf_router_balance_bwd(l, ex, n, g, X, m, T, D, E, 1.0, 0.0, d, dX, dm, w, wb, None)
    assert bwd(D=60) == bwd(D=0) == bwd(E=17) == bwd(T=1 << 29) == SF_ERR_SHAPE
    assert bwd(l=NONE) == bwd(ex=NONE) == bwd(n=NONE) == bwd(X=NONE) == bwd(m=NONE) == bwd(w=NONE) == SF_ERR_NULL
    assert bwd(X=ODD) == bwd(m=ODD) == bwd(d=ODD) == bwd(dX=ODD) == bwd(dm=ODD) == bwd(w=ODD) == bwd(g=C.c_void_p(0x10002)) == SF_ERR_ALIGN
    assert bwd(wb=need - 1) == SF_ERR_WORKSPACE
    assert bwd(dX=AT[4]) == bwd(dm=AT[5]) == bwd(dX=AT[8]) == bwd(w=AT[4]) == bwd(dm=AT[6]) == bwd(dX=C.c_void_p((7 << 36) + 16)) == SF_ERR_UNSUPPORTED
    assert bwd(dX=NONE, dm=NONE, l=NONE) == SF_OK


def test_orthogonalize(lib):
    need = binding.sf_orthogonalize_workspace_size(33, 70)
    abc = (3.4445, -4.7750, 2.0315)
    def run(G=AT[0], type=0, rows=33, cols=70, ldg=70, steps=5, abc=abc, O=AT[1], ldo=70, w=AT[2], wb=need):
        return lib.sf_orthogonalize(G, type, rows, cols, ldg, steps, *abc, 1.0, O, ldo, w, wb, None)
    assert run(rows=-1) == run(cols=(1 << 24) + 1) == run(rows=(1 << 16) + 1, cols=(1 << 16) + 1) == SF_ERR_SHAPE
    assert run(type=2) == run(steps=0) == run(steps=65) == SF_ERR_UNSUPPORTED
    assert run(abc=(3.4445, -4.0, 2.0315)) == run(abc=(9.0, -8.0, 1.0)) == run(abc=(float("nan"), 0, 0)) == run(abc=(1.5, 0.0, 0.0)) == SF_ERR_UNSUPPORTED
    assert run(G=NONE) == run(O=NONE) == run(w=NONE) == SF_ERR_NULL
    assert run(ldg=69) == run(ldo=69) == run(G=C.c_void_p(0x10001)) == run(type=1, G=C.c_void_p(0x10002)) == run(O=C.c_void_p(0x10001)) == run(w=ODD) == SF_ERR_ALIGN
    assert run(wb=need - 1) == SF_ERR_WORKSPACE
    assert run(O=AT[0]) == run(w=AT[0]) == run(O=AT[2]) == SF_ERR_UNSUPPORTED
    assert run(rows=0, G=NONE) == run(cols=0, G=NONE, ldg=0, ldo=0) == SF_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a device")
def test_cpu_tensors_are_refused(lib):
    z = torch.zeros
    X, g = z((4, 64), dtype=torch.bfloat16), z(64, dtype=torch.bfloat16)
    for call in (lambda: binding.sf_rmsnorm_fwd(X, g, 1e-6, Y=z((4, 64), dtype=torch.bfloat16)),
                 lambda: binding.sf_rmsnorm_bwd(X, X, g, z(4), dX=z((4, 64), dtype=torch.bfloat16)),
                 lambda: binding.sf_orthogonalize(X, out=z((4, 64), dtype=torch.bfloat16), workspace=z(10, dtype=torch.uint8))):
        with pytest.raises(binding.SparseFFNError) as e:
            call()
        assert e.value.status == SF_ERR_UNSUPPORTED


def test_wrong_types_and_shapes_are_refused(lib):
    """Found from the tensors, before a pointer of them is used."""
    bf, z = torch.bfloat16, torch.zeros
    X, g = z((4, 64), dtype=bf), z(64, dtype=bf)
    cases = [lambda: binding.sf_rmsnorm_fwd(X.float(), g, 1e-6, Y=X), lambda: binding.sf_rmsnorm_fwd(X, g[:60], 1e-6, Y=X),
             lambda: binding.sf_rmsnorm_fwd(X, g, 1e-6, residual=X[:2], Y=X), lambda: binding.sf_rmsnorm_fwd(X, g, 1e-6, codes=X),
             lambda: binding.sf_rmsnorm_bwd(X, X, g, z(4, dtype=bf), dX=X),
             lambda: binding.sf_gemm_fp8_rows(X, z(4), X, 1.0, C_out=X, workspace=z(256, dtype=torch.uint8)),
             lambda: binding.sf_router_balance_fwd(X, z(4, dtype=torch.int32), 1.0, loss=z(3), counts=z(64, dtype=torch.int32), workspace=z(9)),
             lambda: binding.sf_router_balance_fwd(z((4, 5)), z(4, dtype=torch.int64), 1.0, loss=z(3), counts=z(5, dtype=torch.int32), workspace=z(9)),
             lambda: binding.sf_orthogonalize(X.half()), lambda: binding.sf_orthogonalize(X, out=z((64, 4), dtype=bf), workspace=X),
             lambda: binding.sf_orthogonalize(X[0])]
    for i, c in enumerate(cases):
        with pytest.raises(binding.SparseFFNError) as e:
            c()
        assert e.value.status == SF_ERR_SHAPE, i
    with pytest.raises(binding.SparseFFNError) as e:
        binding.sf_orthogonalize(X.T, out=z((64, 4), dtype=bf), workspace=z(9))
    assert e.value.status == SF_ERR_ALIGN


def test_gradients_of_the_balance_loss_drain_their_copies_after_an_expired_wait():
    """As for the products' kernels: a CTA that gave up a wait lets the copies into its shared memory land before it leaves, and says so."""
    import os
    text = open(os.path.join(build.CSRC, "balance_grad.cuh")).read()
    body = text[text.index("\nbalance_grad_kernel("):]
    body = body[:body.index("\n}\n")]
    assert "tma_load_2d(" in body and "drain_after_expiry()" in body and "atomicExch(a.status, 1)" in body
    assert body.index("pdl_wait()") < body.index("mbar_wait_warp(")          # a wait's budget begins behind the launch before
