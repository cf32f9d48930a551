"""The oracle of the norm, the balance loss and the orthogonalised update: gradients against differences, closed forms, identities."""
import numpy as np
import pytest

from oracle import around


def _rng(*seed):
    return np.random.default_rng(seed)


def _bf(x):
    return around.rne_bf16(x)


@pytest.mark.parametrize("T,D", [(1, 8), (5, 24), (7, 64)])
def test_norm_gradients_against_differences(T, D):
    r = _rng(T, D)
    S, gamma, dY, dS = _bf(r.normal(size=(T, D))), _bf(1 + 0.1 * r.normal(size=D)), r.normal(size=(T, D)), r.normal(size=(T, D))
    eps, h = 1e-5, 1e-6

    def value(s, g):                                         # (without the storage rounding, which has no derivative)
        return np.sum(dY * (s / np.sqrt(np.mean(s * s, axis=1, keepdims=True) + eps) * g)) + np.sum(dS * s)
    _, rs, y = around.rmsnorm_fwd(S, None, gamma, eps)
    dX, dg = around.rmsnorm_bwd(dY, S, rs, gamma, dS)
    assert np.allclose(y, S * rs * gamma)
    for _ in range(6):
        v, w = r.normal(size=S.shape), r.normal(size=D)
        assert np.isclose((value(S + h * v, gamma) - value(S - h * v, gamma)) / (2 * h), np.sum(dX * v), rtol=1e-6, atol=1e-6)
        assert np.isclose((value(S, gamma + h * w) - value(S, gamma - h * w)) / (2 * h), np.sum(dg * w), rtol=1e-6, atol=1e-6)


def test_norm_rows_have_unit_size_and_the_sum_is_rounded():
    r = _rng(3)
    x, res = _bf(r.normal(size=(9, 256)) * 7), _bf(r.normal(size=(9, 256)))
    S, _, y = around.rmsnorm_fwd(x, res, np.ones(256), 0.0)
    assert np.allclose(np.mean(y * y, axis=1), 1) and np.array_equal(S, _bf(x + res)) and not np.array_equal(S, x + res)


@pytest.mark.parametrize("T,E,cb,cz", [(1, 1, 1.0, 0.5), (12, 5, 0.3, 0.0), (40, 16, 0.0, 0.7), (33, 8, 0.2, 0.1)])
def test_balance_gradients_against_differences(T, E, cb, cz):
    r = _rng(T, E)
    D = 16
    X, means = r.normal(size=(T, D)), r.normal(size=(E, D)) * 0.4
    expert = np.argmax(X @ means.T, axis=1)
    expert[T // 2:T // 2 + 2] = -1
    dX, dm, _ = around.balance_bwd(X @ means.T, expert, cb, cz, X, means, dloss=2.0)
    h = 1e-6

    def value(x, m):
        return 2.0 * around.balance_fwd(x @ m.T, expert, cb, cz)[0][0]
    for _ in range(6):
        v, w = r.normal(size=X.shape), r.normal(size=means.shape)
        assert np.isclose((value(X + h * v, means) - value(X - h * v, means)) / (2 * h), np.sum(dX * v), rtol=1e-5, atol=1e-7)
        assert np.isclose((value(X, means + h * w) - value(X, means - h * w)) / (2 * h), np.sum(dm * w), rtol=1e-5, atol=1e-7)


def test_balance_of_even_and_of_single_use():
    E, T = 4, 32
    even = np.tile(np.arange(E), T // E)
    b, n = around.balance_fwd(np.zeros((T, E)), even, 1.0, 0.0)
    assert np.isclose(b[1], 1) and np.isclose(b[0], 1) and np.array_equal(n, np.full(E, T // E))
    sure = np.zeros((T, E))
    sure[:, 2] = 1000.0
    b, n = around.balance_fwd(sure, np.full(T, 2), 1.0, 0.0)
    assert np.isclose(b[1], E) and np.array_equal(n, [0, 0, T, 0])
    b, n = around.balance_fwd(sure, np.full(T, E), 1.0, 1.0)
    assert np.array_equal(b, np.zeros(3)) and n.sum() == 0
    dX, dm, dl = around.balance_bwd(sure, np.full(T, -1), 1.0, 1.0, np.full((T, 8), np.nan), np.ones((E, 8)))
    assert not dl.any() and not dm.any() and not dX.any()


@pytest.mark.parametrize("m,n", [(1, 5), (5, 1), (12, 12), (16, 40), (40, 16)])
def test_orthogonalize_acts_on_singular_values(m, n):
    G = _rng(m, n).normal(size=(m, n))
    assert np.allclose(around.orthogonalize(G), around.orthogonalize_svd(G), atol=1e-10)
    assert np.allclose(around.orthogonalize(G * 1e-20), around.orthogonalize(G), atol=1e-10)
    assert not around.orthogonalize(G * 0).any()


def test_roundings_of_the_product_path_are_small():
    """What keeps the operands' roundings from growing: the second term of X and the diagonals apart (low rank and equal values are where
    they would)."""
    r = _rng(7)
    low = _bf(r.normal(size=(128, 8)) @ r.normal(size=(8, 320)))
    for G in (_bf(r.normal(size=(128, 320))), low, _bf(r.normal(size=(96, 96))), _bf(r.normal(size=(8, 2000)))):
        e = around.orthogonalize(G)
        assert np.linalg.norm(around.orthogonalize_rounded(G) - e) < 2.5e-3 * np.linalg.norm(e)
