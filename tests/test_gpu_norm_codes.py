"""E4M3 codes of the norm with a scale to every row, bit for bit: r falls out of y / scale, so that a code is that of 448 S gamma / max |S gamma|, S and
gamma bf16. Many of these quotients are exactly half-way between two codes, and the even one is the right one. 64 bits hold the quotient well enough: 19 bits
over 16 that are no such half are 2^-21 away from it at least."""
import numpy as np
import pytest
import torch

from oracle import around, f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import f32, to_dev

pytestmark = pytest.mark.gpu
E4 = torch.float8_e4m3fn


def _dev(a):
    return to_dev(f32_to_bf16(np.asarray(a, np.float32)).reshape(a.shape))


def _e4m3(v):
    """The nearest value, ties to even; and whether it was a tie."""
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -20))), -6) - 3)
    return np.rint(v / step) * step, np.abs(np.abs(v / step) % 1 - 0.5) == 0


def _codes(S, gamma, eps):
    T, D = S.shape
    codes, scales = torch.zeros((T, D), dtype=torch.uint8, device="cuda"), torch.zeros(T, device="cuda")
    b.sf_rmsnorm_fwd(_dev(S), _dev(gamma), eps, codes=codes, scales=scales)
    return codes, scales


def _check(S, gamma, eps):
    p = S * gamma
    want, ties = _e4m3(448 * p / np.max(np.abs(p), axis=1, keepdims=True))
    codes, scales = _codes(S, gamma, eps)
    got = f32(codes.view(E4)).astype(np.float64)
    assert np.array_equal(got, want), (int((got != want).sum()), int(ties.sum()), np.argwhere(got != want)[0])
    y = around.rmsnorm_fwd(S, None, gamma, eps)[2]
    assert np.allclose(scales.cpu().numpy(), np.max(np.abs(y), axis=1) / 448, rtol=2.0 ** -16)
    return int(ties.sum())


# every way in which a row is cut over threads: less than a warp, one, two and four vectors to a thread, few rows and many
SHAPES = [(3, 64), (40, 128), (2, 264), (1, 8200), (148, 16384), (200, 512), (300, 4104), (150, 32768)]


@pytest.mark.parametrize("T,D", SHAPES)
def test_small_integers(T, D):
    """The largest is 256 in every row: quotients are halves of a code's step all over."""
    r = np.random.default_rng([T, D])
    S, gamma = r.integers(-63, 64, size=(T, D)).astype(np.float64), 2.0 ** r.integers(-3, 1, size=D)
    gamma[:2], S[:, 0], S[:, 1] = 1.0, 64.0, -7.0
    assert _check(S, gamma, 1e-6) > 0


@pytest.mark.parametrize("T,D", SHAPES)
def test_normal_rows(T, D):
    r = np.random.default_rng([T, D, 1])
    _check(around.rne_bf16(r.normal(size=(T, D)) * 2.0 ** r.normal(size=(T, 1))), around.rne_bf16(1 + 0.1 * r.normal(size=D)), 1e-5)


@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 40])
@pytest.mark.parametrize("weight", [2.0 ** -60, 2.0 ** 100])
def test_sizes_do_not_matter(size, weight):
    """Powers of two leave the codes as they are, as long as the largest |y| is not below 2^-96."""
    r = np.random.default_rng(7)
    S, gamma = around.rne_bf16(r.normal(size=(20, 1032))), around.rne_bf16(1 + 0.1 * r.normal(size=1032))
    _check(S * size, gamma * weight, 0.0)
    assert torch.equal(_codes(S * size, gamma * weight, 0.0)[0], _codes(S, gamma, 0.0)[0])


def test_rows_below_the_least_scale():
    """A row whose largest |y| is below 2^-96 is scaled by that: its codes are those of y * (448 / 2^-96), the float32 error of y allowed for."""
    r = np.random.default_rng(8)
    S, gamma = around.rne_bf16(r.normal(size=(6, 520))), around.rne_bf16(1 + 0.1 * r.normal(size=520)) * 2.0 ** -100
    codes, scales = _codes(S, gamma, 0.0)
    y = around.rmsnorm_fwd(S, None, gamma, 0.0)[2]
    assert np.all(scales.cpu().numpy() == np.float32(2.0 ** -96) / np.float32(448))
    v, got = y * (448 * 2.0 ** 96), f32(codes.view(E4)).astype(np.float64)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -20))), -6) - 3)
    assert np.abs(got).max() > 30 and np.all(np.abs(got - v) <= step / 2 + 2.0 ** -16 * np.abs(v))
