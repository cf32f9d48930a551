"""What stands around the feed-forward layer in a step: the root-mean-square norm with the residual's sum, the router's balance loss, and
the orthogonalised update. Test infrastructure only; float64, from the formulas, with the storage roundings that are part of a definition.
"""
import numpy as np

from .gated import rne_bf16


# ---- norm -------------------------------------------------------------------------------------------------
def rmsnorm_fwd(x, residual, gamma, eps):
    """(S, r, y): the sum as it is stored, 1 / rms of its rows, the normalised rows."""
    S = rne_bf16(x if residual is None else x + residual)
    with np.errstate(all="ignore"):
        r = 1 / np.sqrt(np.mean(S * S, axis=1, keepdims=True) + eps)
        return S, r, S * r * gamma


def rmsnorm_bwd(dY, S, r, gamma, dS=None):
    """(dX, dgamma)."""
    n, q = S * r, dY * gamma
    dX = r * (q - n * np.mean(q * n, axis=1, keepdims=True))
    return dX + (0 if dS is None else dS), np.sum(dY * n, axis=0)


# ---- balance ------------------------------------------------------------------------------------------------
def softmax(l):
    with np.errstate(all="ignore"):
        top = np.max(l, axis=1, keepdims=True)
        e = np.exp(l - top)
        z = np.sum(e, axis=1, keepdims=True)
        return e / z, (top + np.log(z))[:, 0]


def balance_fwd(logits, expert, cb, cz):
    """((loss, balance, z), counts)."""
    E = logits.shape[1]
    here = (expert >= 0) & (expert < E)
    counts = np.bincount(expert[here], minlength=E)[:E]
    n = int(here.sum())
    if n == 0:
        return np.zeros(3), counts
    p, lse = softmax(logits[here])
    b = E * np.sum(counts / n * (np.sum(p, axis=0) / n))
    z = np.mean(lse * lse)
    return np.array([cb * b + cz * z, b, z]), counts


def balance_bwd(logits, expert, cb, cz, X, means, dloss=1.0, dX_in=None):
    """(dX, dmeans, dl). A token that is left out has dl = 0 and its X is not looked at."""
    T, E = logits.shape
    here = (expert >= 0) & (expert < E)
    counts = np.bincount(expert[here], minlength=E)[:E]
    n = max(int(here.sum()), 1)
    dl = np.zeros((T, E))
    if here.any():
        p, lse = softmax(logits[here])
        dl[here] = dloss * p * (cb * E / n ** 2 * (counts - p @ counts[:, None]) + (2 * cz / n * lse)[:, None])
    dX = dl @ means + (0 if dX_in is None else dX_in)
    return dX, dl[here].T @ X[here], dl


# ---- orthogonalised update -------------------------------------------------------------------------------------
ABC = (3.4445, -4.7750, 2.0315)


def orthogonalize(G, steps=5, abc=ABC, scale=1.0):
    """By the iteration itself."""
    a, b, c = abc
    X = G if G.shape[0] <= G.shape[1] else G.T
    norm = np.linalg.norm(X)
    X = X / norm if norm > 0 else X * 0
    for _ in range(steps):
        A = X @ X.T
        X = a * X + (b * A + c * A @ A) @ X
    return scale * (X if G.shape[0] <= G.shape[1] else X.T)


def orthogonalize_svd(G, steps=5, abc=ABC):
    """By what it means: every singular value through the quintic, the vectors as they are."""
    a, b, c = abc
    u, s, vt = np.linalg.svd(G, full_matrices=False)
    s = s / np.linalg.norm(s)
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (u * s) @ vt


def _f16(x):
    return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def orthogonalize_rounded(G, steps=5, abc=ABC):
    """With the operands' roundings of the product path: fp16 numbers (2^14 X in two terms, the first in the products; 2^14 A and 2^12 B
    without their diagonals, which are exact), everything else exact. How far this is from ``orthogonalize`` is what those roundings do; the
    float32 sums of the product path make some of them fall the other way, which is as large at most."""
    a, b, c = abc
    X = G if G.shape[0] <= G.shape[1] else G.T
    norm = np.linalg.norm(X)
    if norm == 0:
        return G * 0
    k = 13 - int(np.floor(np.log2(norm)))
    x, f = X * 2.0 ** k, 2.0 ** 14 / (norm * 2.0 ** k)
    hi = _f16(x)
    lo = _f16(x - hi)
    for _ in range(steps):
        A = hi @ hi.T * f * f * 2.0 ** -28
        D = np.diag(A).copy()
        Ap = _f16((A - np.diag(D)) * 2.0 ** 14) * 2.0 ** -14
        sq = Ap @ Ap
        diag = a + b * D + c * (D * D + np.diag(sq))
        Bp = b * Ap + c * (sq + (D[:, None] + D[None, :]) * Ap)
        Bp = _f16((Bp - np.diag(np.diag(Bp))) * 2.0 ** 12) * 2.0 ** -12
        y = f * (diag[:, None] * (hi + lo) + Bp @ hi)
        f = 1.0
        hi = _f16(y)
        lo = _f16(y - hi)
    y = y * 2.0 ** -14
    return y if G.shape[0] <= G.shape[1] else y.T
