"""Orthogonalised updates of matrices that are far from full rank, wide ones of 512 rows and more among them, as a batch of fewer tokens than rows
leaves them: where G has no component, a step brings up 3.4 times what rounding puts there.

Bound, in the 2-norm: 1.1 times what rounding the exact result to bf16 does (with few different values in it: half a step, 2^-8), and twice
what the operands' roundings do, which the oracle computes by making them."""
import numpy as np
import pytest
import torch

from oracle import around, f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import f32, to_dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _matrix(kind, m, n):
    r = np.random.default_rng([m, n])
    normal, bf = r.normal, around.rne_bf16
    if kind.startswith("rank"):
        k = int(kind[4:])
        return bf(normal(size=(m, k)) @ normal(size=(k, n)))
    if kind == "spike":                                    # one direction, and noise that is 16000 times smaller
        return bf(np.outer(normal(size=m), normal(size=n)) + 6e-5 * normal(size=(m, n)))
    if kind.startswith("copies"):                          # of so many different rows
        k = int(kind[6:])
        return np.tile(bf(normal(size=(k, n))), (-(-m // k), 1))[:m]
    if kind == "ones":
        return np.ones((m, n))
    f = np.arange(1, 257) ** -0.5                          # "full": some directions carry most of it, the rest is spread over all
    return bf((normal(size=(m, 256)) * f) @ normal(size=(256, n)) + 0.3 * normal(size=(m, n)))


def _check(kind, m, n, dtype=BF, steps=5, abc=around.ABC, high=False):
    G = _matrix(kind, m, n)
    if dtype is torch.float32 and not kind.startswith(("copies", "ones")):
        G = (G * (1 + 1e-4 * np.random.default_rng(m).normal(size=G.shape))).astype(np.float32).astype(np.float64)
    want = around.orthogonalize(G, steps, abc)
    made = np.linalg.norm(around.orthogonalize_rounded(G, steps, abc) - want)
    size = np.linalg.norm(want)
    once = 2.0 ** -8 * size if kind == "ones" else 1.1 * np.linalg.norm(around.rne_bf16(want) - want)
    t = torch.from_numpy(np.ascontiguousarray(G.T if high else G, dtype=np.float32)).cuda().to(dtype)
    got = f32(b.sf_orthogonalize(t, steps, abc)).astype(np.float64)
    off = np.linalg.norm((got.T if high else got) - want)
    assert off <= once + 2 * made, (off / size, once / size, made / size)
    assert made < 1e-2 * size                              # the bound is one


KINDS = ["rank1", "rank8", "rank64", "rank256", "spike", "copies1", "copies8", "copies64", "ones"]


@pytest.mark.parametrize("kind", KINDS)
def test_wide(kind):
    _check(kind, 520, 6800)


@pytest.mark.parametrize("kind", ["rank64", "spike", "copies8"])
def test_high_and_in_32_bits(kind):
    _check(kind, 520, 6800, torch.float32, high=True)


@pytest.mark.parametrize("kind", ["rank1", "rank256", "copies8", "full"])
def test_larger(kind):
    _check(kind, 1030, 7300)


@pytest.mark.parametrize("kind", ["rank8", "copies8", "ones"])
@pytest.mark.parametrize("m,n", [(40, 300), (120, 1024), (200, 320)])
def test_small(kind, m, n):
    """In one launch, and in several."""
    _check(kind, m, n)


@pytest.mark.parametrize("steps,abc", [(1, around.ABC), (2, around.ABC), (8, around.ABC), (9, (2.0, -1.5, 0.5)), (7, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0)),
                                       (5, (4.0, -8.0, 3.5))])
def test_steps_and_quintics(steps, abc):
    _check("full", 520, 6800, steps=steps, abc=abc)
    if abc[0] < 3:                                         # quintics that are gentle with what rounding leaves
        _check("rank64", 520, 6800, steps=steps, abc=abc)
