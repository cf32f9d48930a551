"""How the gated block's products are cut (host arithmetic): every form is taken by some shape of the GPU tests, and no plan asks for
what its kernel does not have."""
import ctypes as C

import pytest

from paper_2602_06183_b200 import binding as b
from paper_2602_06183_b200 import build
from test_gpu_gated import FORM_SHAPES, SHAPES


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()
    return b.lib()


def _plan(T, D, F):
    p = b.sf_gated_ffn_step_plan(b.make_gated_desc(T, D, F))
    return [(p.form[i], p.cols[i], p.parts[i]) for i in range(6)]


def test_every_form_of_every_product_is_tested():
    taken = set()
    for s in SHAPES + FORM_SHAPES:
        for i, (form, cols, parts) in enumerate(_plan(*s)):
            taken.add((i, form, cols if form == b.SF_GATED_FEW else cols == 256))
    want = {(i, form, full) for i in range(6) for form in (b.SF_GATED_TILES, b.SF_GATED_SPLIT) for full in (False, True)}
    want |= {(i, b.SF_GATED_FEW, n) for i in range(5) for n in (16, 32, 64, 96, 128)}
    assert want <= taken, sorted(want - taken)


@pytest.mark.parametrize("T", [1, 15, 16, 17, 64, 96, 97, 128, 129, 256, 1000, 8192, 100_000])
@pytest.mark.parametrize("D,F", [(8, 8), (64, 4096), (1408, 5504), (4096, 16384), (8192, 28672), (28672, 72)])
def test_plans_stay_within_their_kernels(T, D, F):
    for i, (form, cols, parts) in enumerate(_plan(T, D, F)):
        blocks = -(-{b.SF_GATED_H: D, b.SF_GATED_H_KEPT: D, b.SF_GATED_Y: F, b.SF_GATED_DH: D, b.SF_GATED_DX: F, b.SF_GATED_DW: T}[i] // 64)
        blocks *= 2 if i == b.SF_GATED_DX else 1
        assert 1 <= parts <= blocks
        if form == b.SF_GATED_FEW:
            assert T <= cols <= 128 and parts <= 8 and i != b.SF_GATED_DW
        else:
            assert cols in range(64, 257, 64 if i < 2 else 32) and parts <= 4
            assert (form == b.SF_GATED_SPLIT) == (parts > 1)


def test_plan_refuses(lib):
    plan = b.sf_gated_ffn_plan()
    assert lib.sf_gated_ffn_step_plan(None, C.byref(plan)) == b.SF_ERR_NULL
    assert lib.sf_gated_ffn_step_plan(C.byref(b.make_gated_desc(4, 64, 64)), None) == b.SF_ERR_NULL
    assert lib.sf_gated_ffn_step_plan(C.byref(b.make_gated_desc(4, 63, 64)), C.byref(plan)) == b.SF_ERR_SHAPE
    assert _plan(0, 64, 64) == [(b.SF_GATED_NONE, 0, 0)] * 6
