"""4-bit products in every form that their sizes can take: which form that is, the host says (no GPU needed); that each is exact, the GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2602_06183_b200 import binding, build
from test_gpu_fp4 import FMT, SHAPES, SIMPLE, _operand, _same
from util import Guarded

# beyond the shapes tested elsewhere: tiles of 256 columns, one and two to a pair; gated ones, four to a pair; 65 to 128 tokens
# with long reductions through both projections
FORM_SHAPES = [(1030, 2056, 2336), (3330, 2312, 1312), (70, 264, 2336), (96, 136, 2592), (97, 72, 2080), (128, 520, 4128)]


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return binding.lib()


@pytest.mark.parametrize("fmt", ["nv", "mx"])
def test_every_form_is_tested(fmt):
    plain, gated = set(), set()
    for s in SHAPES + FORM_SHAPES:
        p, g = binding.sf_gemm_fp4_plan(*s, FMT[fmt]), binding.sf_gemm_fp4_plan(*s, FMT[fmt], gated=True)
        plain.add((p.form, p.cols, p.parts if p.form == binding.SF_GATED_SPLIT else 1))
        gated.add((g.form, g.cols))
    few = {(binding.SF_GATED_FEW, n) for n in (16, 32, 64, 96, 128)}
    want = {(f, n, 1) for f, n in few} | {(binding.SF_GATED_TILES, n, 1) for n in (128, 256)} | {(binding.SF_GATED_SPLIT, 128, n) for n in (2, 3, 4)}
    assert plain == want, (sorted(want - plain), sorted(plain - want))
    assert gated == few | {(binding.SF_GATED_TILES, 256)}


def test_plan_refuses(lib):
    plan = binding.sf_fp4_plan()
    q = lambda M=4, N=64, K=64, fmt=0, p=C.byref(plan): lib.sf_gemm_fp4_plan(M, N, K, fmt, 0, p)   # noqa: E731
    assert q(N=60) == binding.SF_ERR_SHAPE and q(K=0) == binding.SF_ERR_SHAPE and q(fmt=2) == binding.SF_ERR_UNSUPPORTED
    assert q(p=None) == binding.SF_ERR_NULL
    assert q(M=0) == binding.SF_OK and (plan.form, plan.cols, plan.parts) == (binding.SF_GATED_NONE, 0, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M,N,K", FORM_SHAPES)
def test_products_are_exact_on_simple_scales(fmt, M, N, K):
    """As at the small sizes: products are multiples of 1/16 below 144, sums of up to 7000 of them are exact in float32."""
    r = np.random.default_rng(M + N + K)
    a, A, As = _operand(M, K, fmt, r, SIMPLE[fmt])
    b, B, Bs = _operand(N, K, fmt, r, SIMPLE[fmt])
    g, G, Gs = _operand(N, K, fmt, r, SIMPLE[fmt][:2])
    out, ws = Guarded((M, N), torch.bfloat16), Guarded(binding.sf_gemm_fp4_workspace_size(M, N, K), zero=True)
    binding.sf_gemm_fp4(A, As, B, Bs, FMT[fmt], 0.25, C_out=out.t, workspace=ws.t)
    assert binding.sf_check_status(ws.t) == binding.SF_OK
    out.check(); ws.check()   # noqa: E702
    _same(out.t, 0.25 * (a @ b.T), "C")
    out.t.zero_()
    binding.sf_gemm_fp4_gated(A, As, G, Gs, B, Bs, FMT[fmt], binding.SF_ACT_RELU, 0.5, 0.25, H_out=out.t, workspace=ws.t)
    assert binding.sf_check_status(ws.t) == binding.SF_OK
    out.check(); ws.check()   # noqa: E702
    # each factor is exact, their float32 product is one rounding and bf16's another
    H = np.maximum(0.5 * (a @ g.T), 0).astype(np.float32) * (0.25 * (a @ b.T)).astype(np.float32)
    _same(out.t, H.astype(np.float64), "H")
