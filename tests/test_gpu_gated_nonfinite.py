"""What is not a number stays visible: a NaN that only the gate meets goes through every activation into all that the gate enters,
forward, backward and on 4-bit operands, and into nothing else."""
import numpy as np
import pytest

from oracle import gated
from paper_2602_06183_b200 import binding, synth
from test_gpu_gated import GRADS, Block, _normals
from util import bits, f32, to_dev

pytestmark = pytest.mark.gpu

# one token, sums of two terms, one term, and both projections beyond the few-token kernel (see test_gated_plan.py for the forms)
TOKENS = [1, 9, 40, 128, 300]


def _pair(T, D, F, act, data, spoil):
    """The block on the data, and on the data with spoil(Wg) for its gate."""
    out = []
    for w in (data[1], spoil(data[1].copy())):
        b = Block(T, D, F, act, data[0], w, *data[2:])
        b.fwd()
        b.bwd()
        b.check()
        out.append(b)
    return out


def _check(clean, got, f, D, F):
    """Feature f is NaN in all that its gate enters; everything that it does not enter has the bits of the clean block."""
    assert np.isnan(f32(got.Y.t)).all() and np.isnan(f32(got.out["dX"].t)).all()
    rest = np.arange(F) != f
    for k, axis in (("dWg", 0), ("dWu", 0), ("dWd", 1)):
        g, c = f32(got.out[k].t), f32(clean.out[k].t)
        assert np.isnan(np.take(g, f, axis)).all(), k
        assert np.array_equal(np.compress(rest, bits(got.out[k].t), axis), np.compress(rest, bits(clean.out[k].t), axis)), k
        assert np.isfinite(c).all(), k


@pytest.mark.parametrize("act", gated.ACTS)
@pytest.mark.parametrize("T", TOKENS)
def test_a_nan_in_the_gate_weights_alone(act, T):
    D, F, f = 136, 264, 133
    data = _normals(T, D, F, T + 3)

    def spoil(w):
        w[f, 17] = np.nan
        return w
    _check(*_pair(T, D, F, act, data, spoil), f, D, F)


@pytest.mark.parametrize("act", ["relu", "sqrelu"])
@pytest.mark.parametrize("T", TOKENS)
def test_a_gate_of_infinity_less_infinity(act, T):
    D, F, f = 72, 136, 5
    data = list(_normals(T, D, F, T + 4))
    data[0][:, 3], data[0][:, 9] = 1.0, 1.0

    def spoil(w):
        w[f, 3], w[f, 9] = np.inf, -np.inf
        return w
    clean, got = _pair(T, D, F, act, data, spoil)
    assert np.isnan(f32(got.Y.t)).all()
    _check(clean, got, f, D, F)


@pytest.mark.parametrize("act", ["relu", "sqrelu"])
@pytest.mark.parametrize("T", TOKENS)
def test_a_gate_of_minus_infinity_is_cut_off(act, T):
    """ReLU is 0 there, and so is its derivative: the feature is as one whose gate is a large negative number."""
    D, F, f = 72, 136, 5
    data = list(_normals(T, D, F, T + 5))
    data[0][:, 3] = 1.0
    blocks = []
    for v in (-2.0 ** 100, -np.inf):
        w = data[1].copy()
        w[f, 3] = v
        b = Block(T, D, F, act, data[0], w, *data[2:])
        b.fwd()
        b.bwd(("dWg", "dWu", "dWd"))                       # (dX = dG Wg meets 0 times the infinite weight)
        b.check()
        blocks.append(b)
    assert np.array_equal(bits(blocks[0].Y.t), bits(blocks[1].Y.t))
    for k in GRADS[1:]:
        assert np.array_equal(bits(blocks[0].out[k].t), bits(blocks[1].out[k].t)), k


@pytest.mark.parametrize("act", gated.ACTS)
@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M", [1, 40, 300])
def test_a_nan_block_of_the_gate_weights(act, fmt, M):
    N, K, f = 264, 320, 131
    code = {"nv": binding.SF_FP4_NV, "mx": binding.SF_FP4_MX}[fmt]
    a = binding.sf_fp4_quantize(to_dev(synth.normal_bf16((M, K), 0, 1, seed=1)), code, 4.0)
    u = binding.sf_fp4_quantize(to_dev(synth.normal_bf16((N, K), 0, 1, seed=2)), code, 8.0)
    x = synth.normal_bf16((N, K), 0, 1, seed=3)
    H = []
    for spoilt in (False, True):
        if spoilt:
            x[f, 100] = 0x7FC0
        g = binding.sf_fp4_quantize(to_dev(x), code, 8.0)
        H.append(binding.sf_gemm_fp4_gated(*a, *g, *u, code, binding.__dict__["SF_ACT_" + act.upper()], 1 / 32, 1 / 32))
    rest = np.arange(N) != f
    assert np.isfinite(f32(H[0])).all() and np.isnan(f32(H[1])[:, f]).all()
    assert np.array_equal(bits(H[1])[:, rest], bits(H[0])[:, rest])
