"""E4M3 products of rows with scales: both kernels and every size of the few-token one, ragged edges, exact sums of small integers, NaN
codes and scales, and everything around the buffers left alone."""
import numpy as np
import pytest
import torch

from oracle import f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import Guarded, assert_close_elementwise, bits, f32

pytestmark = pytest.mark.gpu
E4 = torch.float8_e4m3fn


def _codes(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(E4).view(torch.uint8).cuda()


def _run(A, s, B, alpha):
    M, K, N = A.shape[0], A.shape[1], B.shape[0]
    C, ws = Guarded((M, N), torch.bfloat16), Guarded(b.sf_gemm_fp8_rows_workspace_size(M, N, K), zero=True)
    assert b.sf_gemm_fp8_rows(A, s, B, alpha, C_out=C.t, workspace=ws.t) is C.t
    assert b.sf_check_status(ws.t) == b.SF_OK
    C.check("C")
    ws.check("workspace")
    return C.t


@pytest.mark.parametrize("M", [1, 2, 16, 17, 32, 33, 64, 65, 96, 97, 128, 129, 255, 513])
@pytest.mark.parametrize("N,K", [(8, 16), (136, 272), (520, 1040)])
def test_small_integers_are_exact(M, N, K):
    """Products and sums of small integers fit float32, and so do scales that are powers of two: only the final rounding is left."""
    r = np.random.default_rng([M, N, K])
    a, w = r.integers(-3, 4, size=(M, K)).astype(np.float64), r.integers(-3, 4, size=(N, K)).astype(np.float64)
    s = 2.0 ** r.integers(-8, 9, size=M)
    C = _run(_codes(a), torch.from_numpy(s.astype(np.float32)).cuda(), _codes(w), 0.25)
    want = (0.25 * s[:, None]) * (a @ w.T)
    assert np.array_equal(bits(C) & 0x7FFF | (bits(C) & 0x8000) * (f32(C) != 0), f32_to_bf16((want + 0.0).astype(np.float32)).reshape(M, N))


@pytest.mark.parametrize("M,N,K", [(1, 4096, 1024), (40, 2048, 4096), (300, 1000, 512), (130, 256, 8192), (2000, 776, 1040), (4096, 4096, 256)])
def test_against_64_bits(M, N, K):
    g = torch.Generator("cuda").manual_seed(M + N + K)
    A, B = ((torch.randn(n, K, generator=g, device="cuda") * 40).clamp(-448, 448).to(E4).view(torch.uint8) for n in (M, N))
    s = torch.rand(M, generator=g, device="cuda") + 0.01
    C = _run(A, s, B, 2.0 ** -11)
    want = 2.0 ** -11 * s.double()[:, None] * (A.view(E4).double() @ B.view(E4).double().T)
    assert_close_elementwise(f32(C), want.cpu().numpy(), K)


@pytest.mark.parametrize("M", [3, 200])
def test_nan_infinity_and_zero(M):
    a, w = np.ones((M, 64)), np.ones((24, 64))
    A, B, s = _codes(a), _codes(w), torch.ones(M, device="cuda")
    A[1, 5] = 0x7F                                       # a NaN code
    s[0], s[2] = 0.0, float("nan")
    C = f32(_run(A, s, B, 1.0))
    assert not C[0].any() and np.isnan(C[1]).all() and np.isnan(C[2]).all() and np.all(C[3:] == 64)
    s[:] = float("inf")
    assert np.all(f32(_run(_codes(a), s, B, 1.0)) == np.inf)


def test_nothing_to_do():
    e = torch.empty
    s0, u8 = torch.zeros(0, device="cuda"), dict(dtype=torch.uint8, device="cuda")
    assert b.sf_gemm_fp8_rows(e((0, 64), **u8), s0, e((16, 64), **u8), 1.0).shape == (0, 16)
    assert b.sf_gemm_fp8_rows(e((3, 64), **u8), torch.zeros(3, device="cuda"), e((0, 64), **u8), 1.0).shape == (3, 0)


def test_a_row_does_not_depend_on_the_others():
    """Within a kernel's range a token's result has the same bits whatever runs beside it."""
    g = torch.Generator("cuda").manual_seed(1)
    A, B = ((torch.randn(n, 512, generator=g, device="cuda")).to(E4).view(torch.uint8) for n in (300, 256))
    s = torch.rand(300, generator=g, device="cuda")
    for M, m in ((16, 3), (300, 200)):
        C = _run(A[:M], s[:M], B, 1.0)
        A2, s2 = A[:M].flip(0).contiguous(), s[:M].flip(0).contiguous()
        assert torch.equal(_run(A2, s2, B, 1.0)[M - 1 - m], C[m])
