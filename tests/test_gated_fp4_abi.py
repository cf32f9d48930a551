"""What the gated block and the 4-bit calls refuse, on the host: nothing is launched (no GPU needed, the pointers are fake)."""
import ctypes as C

import pytest
import torch

from paper_2602_06183_b200 import binding, build
from paper_2602_06183_b200.binding import (SF_ERR_ALIGN, SF_ERR_NULL, SF_ERR_SHAPE, SF_ERR_UNSUPPORTED, SF_ERR_WORKSPACE, SF_OK)

P, ODD, NONE = C.c_void_p(0x10000), C.c_void_p(0x10008), None


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def test_gated_sizes(lib):
    ctx, ws = binding.sf_gated_ffn_workspace_size(binding.make_gated_desc(100, 64, 72))
    assert ctx >= 100 * 72 * 10 and ws >= 256 + 2 * 100 * 72 * 2
    assert binding.sf_gated_ffn_workspace_size(binding.make_gated_desc(0, 64, 72))[1] == 256
    a, b = C.c_size_t(), C.c_size_t()
    for T, D, F, act, want in [(-1, 64, 64, 0, SF_ERR_SHAPE), (4, 60, 64, 0, SF_ERR_SHAPE), (4, 64, 63, 0, SF_ERR_SHAPE),
                               (4, 0, 64, 0, SF_ERR_SHAPE), (4, 64, 64, 5, SF_ERR_UNSUPPORTED), (4, 64, 64, -1, SF_ERR_UNSUPPORTED),
                               (1 << 29, 64, 64, 0, SF_ERR_SHAPE), (4, 1 << 29, 64, 0, SF_ERR_SHAPE)]:
        assert lib.sf_gated_ffn_workspace_size(C.byref(binding.make_gated_desc(T, D, F, act)), C.byref(a), C.byref(b)) == want
    assert lib.sf_gated_ffn_workspace_size(None, C.byref(a), C.byref(b)) == SF_ERR_NULL
    assert lib.sf_gated_ffn_workspace_size(C.byref(binding.make_gated_desc(4, 64, 64)), None, C.byref(b)) == SF_ERR_NULL


def test_gated_calls_refuse_before_launching(lib):
    d = binding.make_gated_desc(16, 64, 128)
    ctx, ws = binding.sf_gated_ffn_workspace_size(d)
    fwd = lambda *, X=P, Wd=P, Y=P, c=P, cb=ctx, w=P, wb=ws: lib.sf_gated_ffn_fwd(C.byref(d), X, P, P, Wd, Y, c, cb, w, wb, None)  # noqa: E731
    assert fwd(X=NONE) == SF_ERR_NULL and fwd(Wd=NONE) == SF_ERR_NULL and fwd(Y=NONE) == SF_ERR_NULL and fwd(w=NONE) == SF_ERR_NULL
    assert fwd(X=ODD) == SF_ERR_ALIGN and fwd(c=ODD) == SF_ERR_ALIGN and fwd(Y=ODD) == SF_ERR_ALIGN
    assert fwd(cb=ctx - 1) == SF_ERR_WORKSPACE and fwd(wb=255) == SF_ERR_WORKSPACE
    assert fwd(c=NONE, cb=0, wb=256 + 2 * 16 * 128 - 1) == SF_ERR_WORKSPACE
    bwd = lambda *, dY=P, c=P, cb=ctx, dX=P, dWg=P, wb=ws: lib.sf_gated_ffn_bwd(C.byref(d), dY, P, P, P, P, c, cb, dX, dWg, P, P, P, wb, None)  # noqa: E731
    assert bwd(dY=NONE) == SF_ERR_NULL and bwd(c=NONE) == SF_ERR_NULL
    assert bwd(dX=ODD) == SF_ERR_ALIGN and bwd(dWg=ODD) == SF_ERR_ALIGN and bwd(c=ODD) == SF_ERR_ALIGN
    assert bwd(cb=ctx - 1) == SF_ERR_WORKSPACE and bwd(wb=ws - 1) == SF_ERR_WORKSPACE
    # nothing asked for, or nothing to do: no pointer is looked at
    assert lib.sf_gated_ffn_bwd(C.byref(d), P, P, P, P, P, P, ctx, None, None, None, None, P, ws, None) == SF_OK
    assert lib.sf_gated_ffn_fwd(C.byref(binding.make_gated_desc(0, 64, 128)), None, None, None, None, None, None, 0, None, 0, None) == SF_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call that were not refused would run on pointers to nothing")
def test_shared_bytes_are_refused(lib):
    """Every buffer far from the others but for the last byte of one and the first of another. (None of these calls gets past the check.)"""
    at = {k: (i + 1) << 30 for i, k in enumerate("X Wg Wu Wd Y c w dY dX dWg dWu dWd".split())}
    T, D, F = 24, 64, 128
    d = binding.make_gated_desc(T, D, F)
    ctx, ws = binding.sf_gated_ffn_workspace_size(d)
    size = dict(X=2 * T * D, Y=2 * T * D, dY=2 * T * D, dX=2 * T * D, c=ctx, w=ws, **{k: 2 * D * F for k in "Wg Wu Wd dWg dWu dWd".split()})

    def run(call, names, n_in):
        for i, a in enumerate(names):
            for b in names[:i]:
                if i < n_in and names.index(b) < n_in:
                    continue                                     # inputs may be one another
                for x, y in ((a, b), (b, a)):                    # x ends on y's first 16 bytes
                    p = dict(at)
                    p[x] = at[y] + 16 - size[x]
                    assert call(*(C.c_void_p(p[k]) for k in names)) == SF_ERR_UNSUPPORTED, (x, y)
    size["w"] = 256                                                  # H lies in the context
    run(lambda X, g, u, dn, Y, c, w: lib.sf_gated_ffn_fwd(C.byref(d), X, g, u, dn, Y, c, ctx, w, ws, None), "X Wg Wu Wd Y c w".split(), 4)
    size["w"] = ws
    run(lambda dY, X, g, u, dn, c, dX, dg, du, dd, w: lib.sf_gated_ffn_bwd(C.byref(d), dY, X, g, u, dn, c, ctx, dX, dg, du, dd, w, ws, None),
        "dY X Wg Wu Wd c dX dWg dWu dWd w".split(), 6)

    at = {k: (i + 1) << 30 for i, k in enumerate("A sa B sb U su C w X c s".split())}
    M, N, K, ld = 130, 72, 96, 104
    size = dict(A=M * K // 2, sa=2 * 2 * 512, B=N * K // 2, sb=2 * 512, U=N * K // 2, su=2 * 512, C=2 * M * N, w=256, c=M * K // 2, s=2 * 2 * 512,
                X=2 * ((M - 1) * ld + K))
    run(lambda A, sa, B, sb, Cc, w: lib.sf_gemm_fp4(A, sa, B, sb, 0, Cc, M, N, K, 1.0, w, 256, None), "A sa B sb C w".split(), 4)
    run(lambda A, sa, B, sb, U, su, Cc, w: lib.sf_gemm_fp4_gated(A, sa, B, sb, U, su, 0, 0, Cc, M, N, K, 1.0, 1.0, w, 256, None),
        "A sa B sb U su C w".split(), 6)
    run(lambda X, c, s: lib.sf_fp4_quantize(X, M, K, ld, 0, 1.0, c, s, None), "X c s".split(), 1)
    run(lambda c, s, X: lib.sf_fp4_dequantize(c, s, M, K, 0, 1.0, X, ld, None), "c s X".split(), 2)


def test_fp4_calls_refuse_before_launching(lib):
    assert binding.sf_fp4_sizes(3, 96, binding.SF_FP4_NV) == (3 * 48, 2 * 512)
    assert binding.sf_fp4_sizes(129, 96, binding.SF_FP4_MX) == (129 * 48, 2 * 512)
    a, b = C.c_size_t(), C.c_size_t()
    assert lib.sf_fp4_sizes(3, 48, 0, C.byref(a), C.byref(b)) == SF_ERR_SHAPE
    assert lib.sf_fp4_sizes(3, 64, 2, C.byref(a), C.byref(b)) == SF_ERR_UNSUPPORTED
    assert lib.sf_fp4_sizes(-1, 64, 0, C.byref(a), C.byref(b)) == SF_ERR_SHAPE
    assert lib.sf_fp4_sizes(3, 64, 0, None, C.byref(b)) == SF_ERR_NULL
    q = lambda *, X=P, rows=4, cols=64, ld=64, fmt=0, c=P, s=P: lib.sf_fp4_quantize(X, rows, cols, ld, fmt, 1.0, c, s, None)  # noqa: E731
    assert q(X=NONE) == SF_ERR_NULL and q(s=NONE) == SF_ERR_NULL and q(cols=40) == SF_ERR_SHAPE and q(fmt=7) == SF_ERR_UNSUPPORTED
    assert q(ld=63) == SF_ERR_ALIGN and q(ld=68) == SF_ERR_ALIGN and q(X=ODD) == SF_ERR_ALIGN and q(c=ODD) == SF_ERR_ALIGN
    assert q(X=NONE, rows=0) == SF_OK
    dq = lambda *, c=P, y=P, ld=64, cols=64: lib.sf_fp4_dequantize(c, P, 4, cols, 1, 1.0, y, ld, None)  # noqa: E731
    assert dq(c=NONE) == SF_ERR_NULL and dq(y=ODD) == SF_ERR_ALIGN and dq(ld=56) == SF_ERR_ALIGN and dq(cols=16) == SF_ERR_SHAPE
    g = lambda *, A=P, sb=P, fmt=0, Cc=P, M=4, N=64, K=64, w=P, wb=256: lib.sf_gemm_fp4(A, P, P, sb, fmt, Cc, M, N, K, 1.0, w, wb, None)  # noqa: E731
    assert g(A=NONE) == SF_ERR_NULL and g(sb=NONE) == SF_ERR_NULL and g(w=NONE) == SF_ERR_NULL and g(fmt=-1) == SF_ERR_UNSUPPORTED
    assert g(N=60) == SF_ERR_SHAPE and g(K=48) == SF_ERR_SHAPE and g(K=0) == SF_ERR_SHAPE and g(M=-1) == SF_ERR_SHAPE
    assert g(Cc=ODD) == SF_ERR_ALIGN and g(sb=ODD) == SF_ERR_ALIGN and g(wb=255) == SF_ERR_WORKSPACE
    assert g(A=NONE, M=0) == SF_OK and g(A=NONE, N=0) == SF_OK
    h = lambda *, u=P, act=0, H=P, wb=256: lib.sf_gemm_fp4_gated(P, P, P, P, u, P, 0, act, H, 4, 64, 64, 1.0, 1.0, P, wb, None)  # noqa: E731
    assert h(u=NONE) == SF_ERR_NULL and h(act=9) == SF_ERR_UNSUPPORTED and h(H=ODD) == SF_ERR_ALIGN and h(wb=0) == SF_ERR_WORKSPACE


def _status(call):
    with pytest.raises(binding.SparseFFNError) as e:
        call()
    return e.value.status


def test_binding_refuses_tensors_that_would_be_read_as_something_else(lib):
    """Shape, type, layout: found before the device is asked for anything (CPU tensors are refused last, as on another device)."""
    bf = torch.bfloat16
    d = binding.make_gated_desc(3, 16, 24)
    X, W, Wd, Y = torch.zeros(3, 16, dtype=bf), torch.zeros(24, 16, dtype=bf), torch.zeros(16, 24, dtype=bf), torch.zeros(3, 16, dtype=bf)
    ws = torch.zeros(4096, dtype=torch.uint8)
    fwd = lambda x=X, w=W, wd=Wd, y=Y: binding.sf_gated_ffn_fwd(d, x, w, W, wd, y, None, ws)   # noqa: E731
    assert _status(lambda: fwd(x=X[:2])) == SF_ERR_SHAPE
    assert _status(lambda: fwd(x=X.float())) == SF_ERR_SHAPE
    assert _status(lambda: fwd(wd=Wd.T)) == SF_ERR_SHAPE
    assert _status(lambda: fwd(w=torch.zeros(24, 32, dtype=bf)[:, ::2])) == SF_ERR_ALIGN
    codes, scales = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    gemm = lambda A=codes, sa=scales, B=codes, fmt=0: binding.sf_gemm_fp4(A, sa, B, scales, fmt, 1.0)   # noqa: E731
    assert _status(lambda: gemm(B=codes[:, :16])) == SF_ERR_SHAPE
    assert _status(lambda: gemm(sa=scales[:256])) == SF_ERR_SHAPE
    assert _status(lambda: gemm(A=codes.view(torch.int8))) == SF_ERR_SHAPE
    assert _status(lambda: gemm(fmt=2)) == SF_ERR_UNSUPPORTED
    assert _status(lambda: binding.sf_gemm_fp4_gated(codes, scales, codes, scales, codes[:2], scales, 0, 0, 1.0, 1.0)) == SF_ERR_SHAPE
    assert _status(lambda: binding.sf_fp4_quantize(torch.zeros(4, 64), 0, 1.0)) == SF_ERR_SHAPE
    assert _status(lambda: binding.sf_fp4_quantize(torch.zeros(64, 4, dtype=bf).T, 0, 1.0)) == SF_ERR_ALIGN
    assert _status(lambda: binding.sf_fp4_quantize(torch.zeros(4, 40, dtype=bf), 0, 1.0)) == SF_ERR_SHAPE
    if not torch.cuda.is_available():
        return
    assert _status(fwd) == SF_ERR_UNSUPPORTED and _status(gemm) == SF_ERR_UNSUPPORTED
    assert _status(lambda: binding.sf_fp4_quantize(torch.zeros(4, 64, dtype=bf), 0, 1.0)) == SF_ERR_UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="a call that were not refused would run on pointers to nothing")
def test_an_infinite_scale_is_refused(lib):
    """x scale would be NaN for every zero of x, which the largest magnitude of a block, taken before the product, does not show."""
    q = lambda scale, rows=4: lib.sf_fp4_quantize(C.c_void_p(1 << 30), rows, 64, 64, 0, scale, C.c_void_p(2 << 30), C.c_void_p(3 << 30), None)   # noqa: E731
    assert q(float("inf")) == SF_ERR_UNSUPPORTED and q(float("-inf")) == SF_ERR_UNSUPPORTED and q(float("inf"), rows=0) == SF_OK
