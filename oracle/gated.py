"""The gated feed-forward block (three matrices; Section 5.1 counts its FLOPs). Test infrastructure only.

    G = X Wg^T,  U = X Wu^T,  H = act(G) * U,  Y = H Wd^T

in float64, with the roundings of the product path where asked for: H, dG and dU are operands of products and are rounded to bf16
once (with up to 16 tokens, to the sum of two bf16 numbers); everything else is not rounded before its end. With the forward values the bounds of their error are
returned too, from the arithmetic alone (see ``forward``).
"""
import math
from dataclasses import dataclass

import numpy as np

from .bf16 import bf16_to_f32, f32_to_bf16

ACTS = ("silu", "gelu", "gelu_tanh", "relu", "sqrelu")
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def act(name, g):
    """(act(g), act'(g)) in float64."""
    if name == "silu":
        s = np.where(g >= 0, 1 / (1 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1 + np.exp(-np.abs(g))))
        return g * s, s + g * s * (1 - s)
    if name == "gelu":
        c = 0.5 * _erfc(-g / math.sqrt(2))
        return g * c, c + g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        z = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        with np.errstate(over="ignore"):
            s, t = 1 / (1 + np.exp(-2 * z)), 1 / (1 + np.exp(2 * z))      # (1 + tanh z) / 2, which cancels below, and (1 - tanh z) / 2
        return g * s, s + 2 * g * s * t * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)
    r = np.maximum(g, 0.0)
    return (r, np.where(np.isnan(g), g, g > 0)) if name == "relu" else (r * r, 2 * r)


def rne_bf16(x):
    """float64 -> nearest bf16 value as float64 (through float32; exact where x is a float32)."""
    return bf16_to_f32(f32_to_bf16(np.asarray(x, np.float64).astype(np.float32))).astype(np.float64)


def two_terms(x):
    """The sum of two bf16 numbers that stands for x: x rounded, and what that left, rounded."""
    hi = rne_bf16(x)
    return hi + rne_bf16(x - hi)


def held(x, T):
    """An operand in between (H, dG, dU): one bf16, or with up to 16 tokens the sum of two."""
    return two_terms(x) if T <= 16 else rne_bf16(x)


U16 = 2.0 ** -8          # a rounding to bf16, relative
ADD = 2.0 ** -23         # an addition in a float32 accumulator, relative to the sum of magnitudes (truncation allowed for)
ELEM = 2.0 ** -20        # an activation's evaluation in float32, relative to (1 + |g|) times its size: a few units of 2^-23 from the
                         # exponential, whose argument's rounding grows with |g|, the quotient and the products


@dataclass
class Gated:
    H: np.ndarray
    Y: np.ndarray
    P: np.ndarray
    Q: np.ndarray
    err_H: np.ndarray
    err_Y: np.ndarray
    err_P: np.ndarray
    err_Q: np.ndarray


def forward(X, Wg, Wu, Wd, name, round_h=True):
    """Float64 values of the block and bounds of what the float32 path may differ by.

    G and U: K additions of products, K 2^-23 of the sum of their magnitudes. P = act(G): |act'| of that plus the evaluation. Q =
    U act'(G): act'' is at most 2 for every act here, but for ReLU, whose derivative steps by 1 at 0. H = P U, rounded
    once. Y: F additions, the error of H, one rounding.
    """
    D, F = X.shape[1], Wg.shape[0]
    G, U = X @ Wg.T, X @ Wu.T
    eg, eu = D * ADD * (np.abs(X) @ np.abs(Wg).T), D * ADD * (np.abs(X) @ np.abs(Wu).T)
    P, dP = act(name, G)
    ep = (np.abs(dP) + 2 * eg) * eg + ELEM * (1 + np.abs(G)) * np.abs(P)
    edp = 2 * eg + ELEM * (1 + np.abs(G)) ** 2
    if name == "relu":
        edp = edp + (np.abs(G) <= eg)        # either side of the step
    Q = U * dP
    eq = (np.abs(dP) + edp) * eu + (np.abs(U) + eu) * edp
    H = P * U
    u = U16 if X.shape[0] > 16 else U16 * U16        # of the operand in between
    eh = (np.abs(P) + ep) * eu + np.abs(U) * ep + u * np.abs(H)
    if round_h:
        H = held(H, X.shape[0])
        eh = eh + u * np.abs(H)          # the reference is rounded too: a value next to a border may go either way
    Y = H @ Wd.T
    ey = eh @ np.abs(Wd).T + F * ADD * (np.abs(H) @ np.abs(Wd).T)
    ey = ey + U16 * (np.abs(Y) + ey)
    return Gated(H, Y, P, Q, eh, ey, ep, eq)


def backward(X, Wg, Wu, Wd, dY, name):
    """{name: (value, bound)} of dX, dWg, dWu, dWd in float64; nothing is rounded here, the bounds count the path's roundings."""
    T, D, F = X.shape[0], X.shape[1], Wg.shape[0]
    f = forward(X, Wg, Wu, Wd, name, round_h=False)
    a = np.abs
    dH = dY @ Wd
    edh = D * ADD * (a(dY) @ a(Wd))
    out = {}
    dU, dG = dH * f.P, dH * f.Q
    edu = (a(f.P) + f.err_P) * edh + a(dH) * f.err_P
    edg = (a(f.Q) + f.err_Q) * edh + a(dH) * f.err_Q
    u = U16 if T > 16 else U16 * U16
    edu, edg = edu + u * (a(dU) + edu), edg + u * (a(dG) + edg)

    def done(v, e):
        return v, e + U16 * (a(v) + e)
    out["dX"] = done(dG @ Wg + dU @ Wu, edg @ a(Wg) + edu @ a(Wu) + 2 * F * ADD * ((a(dG) + edg) @ a(Wg) + (a(dU) + edu) @ a(Wu)))
    out["dWg"] = done(dG.T @ X, edg.T @ a(X) + T * ADD * ((a(dG) + edg).T @ a(X)))
    out["dWu"] = done(dU.T @ X, edu.T @ a(X) + T * ADD * ((a(dU) + edu).T @ a(X)))
    out["dWd"] = done(dY.T @ f.H, a(dY).T @ f.err_H + T * ADD * (a(dY).T @ (a(f.H) + f.err_H)))
    return out


def exact_step(X, Wg, Wu, Wd, dY, name="relu"):
    """Every output of a step whose sums are exact in float32 (small integers, ReLU or its square): the values are those of
    any order of additions, with one rounding to bf16 where the path has one."""
    G, U = X @ Wg.T, X @ Wu.T
    P, dP = act(name, G)
    T = X.shape[0]
    H = held(P * U, T)
    dH = dY @ Wd
    dU, dG = held(dH * P, T), held(dH * (U * dP), T)
    return {"Y": rne_bf16(H @ Wd.T), "dX": rne_bf16(dG @ Wg + dU @ Wu), "dWg": rne_bf16(dG.T @ X), "dWu": rne_bf16(dU.T @ X),
            "dWd": rne_bf16(dY.T @ H)}
