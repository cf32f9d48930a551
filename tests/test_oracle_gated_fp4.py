"""The gated block's and the 4-bit formats' oracles against what they can be checked by: differences, hand-worked values, brute force."""
import numpy as np
import pytest

from oracle import fp4, gated
from oracle.bf16 import f32_to_bf16


def _inputs(T, D, F, seed=0):
    r = np.random.default_rng(seed)
    return [r.normal(size=s) * k for s, k in (((T, D), 1.0), ((F, D), 0.4), ((F, D), 0.4), ((D, F), 0.4), ((T, D), 1.0))]


@pytest.mark.parametrize("name", gated.ACTS)
def test_derivative_of_the_activation_is_its_difference(name):
    g = np.array([-30.0, -9.0, -3.0, -1.2, -0.3, 0.2, 0.9, 2.5, 8.0, 30.0])
    h = 1e-6
    d = (gated.act(name, g + h)[0] - gated.act(name, g - h)[0]) / (2 * h)
    # central differences: h^2 times a third derivative of at most a few, and 2^-52 |act| / h of rounding
    assert np.all(np.abs(d - gated.act(name, g)[1]) <= 1e-10 * 5 + 2.0 ** -51 * (1 + np.abs(gated.act(name, g)[0])) / h)


@pytest.mark.parametrize("name", gated.ACTS)
def test_backward_is_the_difference_of_forward(name):
    X, Wg, Wu, Wd, dY = _inputs(3, 5, 4, seed=1)
    grads = gated.backward(X, Wg, Wu, Wd, dY, name)
    args = {"dX": X, "dWg": Wg, "dWu": Wu, "dWd": Wd}
    loss = lambda: float((gated.forward(X, Wg, Wu, Wd, name, round_h=False).Y * dY).sum())   # noqa: E731
    h = 1e-5
    for k, p in args.items():
        for i in np.ndindex(p.shape):
            old = p[i]
            p[i] = old + h; hi = loss()   # noqa: E702
            p[i] = old - h; lo = loss()   # noqa: E702
            p[i] = old
            assert abs((hi - lo) / (2 * h) - grads[k][0][i]) < 1e-6 * max(1.0, abs(grads[k][0][i]))


@pytest.mark.parametrize("name", gated.ACTS)
def test_a_gate_that_is_not_a_number_stays_one(name):
    P, dP = gated.act(name, np.array([np.nan, -1.0, 2.0]))
    assert np.isnan(P).tolist() == [True, False, False] and np.isnan(dP).tolist() == [True, False, False]


def test_e2m1_ties_and_clamping():
    y = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0001, 7.0, np.inf, -0.25, -0.75, -9.0], np.float32)
    want = [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, 6.0, -0.0, -1.0, -6.0]
    assert fp4.e2m1_to_f64(fp4.f32_to_e2m1(y)).tolist() == want


def test_blocks_by_hand():
    x = np.zeros((1, 32), np.float32)
    x[0, :4] = [12.0, -3.0, 1.0, 0.4]                # nv: sf = 2
    x[0, 16:18] = [0.75, 0.5]                        # nv: sf = 0.125
    codes, by = fp4.quantize(f32_to_bf16(x), "nv", 1.0)
    assert fp4.scale_value(by, "nv").tolist() == [[2.0, 0.125]]
    assert fp4.values(codes, by, "nv")[0, [0, 1, 2, 3, 16, 17]].tolist() == [12.0, -3.0, 1.0, 0.0, 0.75, 0.5]
    codes, by = fp4.quantize(f32_to_bf16(x), "mx", 1.0)
    assert by.tolist() == [[127 + 3 - 2]]            # floor(log2 12) = 3
    assert fp4.values(codes, by, "mx")[0, [0, 1, 2, 3, 16]].tolist() == [12.0, -3.0, 1.0, 0.0, 1.0]


def test_zero_infinite_and_nan_blocks():
    x = np.zeros((1, 64), np.float32)
    x[0, 16], x[0, 17] = np.inf, -1.0
    x[0, 32], x[0, 33] = np.nan, 1.0
    codes, by = fp4.quantize(f32_to_bf16(x), "nv", 1.0)
    assert fp4.scale_value(by, "nv")[0, :2].tolist() == [0.0, 448.0] and np.isnan(fp4.scale_value(by, "nv")[0, 2])
    v = fp4.values(codes, by, "nv")
    assert v[0, 16] == 6 * 448 and v[0, 17] == 0 and np.isnan(v[0, 32:48]).all() and not v[0, :16].any()


def test_tiles_hold_every_scale_once():
    off = fp4.tile_offsets(300, 12)
    assert len(np.unique(off)) == off.size and off.max() < 3 * 3 * 512
    assert fp4.tile_offsets(1, 5)[0].tolist() == [0, 1, 2, 3, 512]
    assert [int(fp4.tile_offsets(129, 4)[r, 0]) for r in (1, 31, 32, 127, 128)] == [16, 496, 4, 508, 512]


def test_quotient_by_reciprocal_and_remainder_is_the_rounded_quotient():
    """What the quantising kernel computes for x / sf: r = 1 / sf rounded down, e = (1 - r sf) r, and x r + x e with one rounding. In
    float64 the sum is exact to 2^-50, so its rounding to float32 is the kernel's result."""
    rng = np.random.default_rng(3)
    sf = fp4.scale_value(np.arange(1, 127, dtype=np.uint8), "nv").astype(np.float32)
    for n in range(20):
        x = np.ldexp(rng.normal(size=4000), rng.integers(-6, 8)).astype(np.float32)
        if n < 10:
            x = (x.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)              # bf16 values
        for s in sf[::5]:
            r = np.float32(1) / s
            if float(r) * float(s) > 1:
                r = np.nextafter(r, np.float32(0))
            e = np.float32(np.float32(1.0 - float(r) * float(s)) * r)
            y = (x.astype(np.float64) * float(r) + (x * e).astype(np.float64)).astype(np.float32)
            assert np.array_equal(y, x / s)
