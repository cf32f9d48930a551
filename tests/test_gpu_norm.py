"""The root-mean-square norm through the C ABI, against the oracle in 64 bits: every way in which a row is cut over threads, the residual in
place, strided rows, 8-bit rows with and without scales, what is not finite, and the backward pass.

Bounds. A row's sum of squares is added up by threads of at most 64 values each and a tree: relative error below 100 x 2^-24, half of it in
1 / rms; with the products' roundings y is within 2^-16 of itself before its last rounding (2^-8 to bf16)."""
import numpy as np
import pytest
import torch

from oracle import around, f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import Guarded, bits, f32, to_dev

pytestmark = pytest.mark.gpu
BF, U16, F32E = torch.bfloat16, 2.0 ** -8, 2.0 ** -16

SHAPES = [(1, 8), (1, 4096), (2, 1032), (5, 64), (3, 32768), (149, 256), (150, 264), (300, 512), (333, 1024), (1000, 1408), (160, 4104),
          (160, 8192), (150, 16384), (152, 32760), (4100, 4104)]
# and of the backward pass: short batches, which one launch takes, and the first ones that take two
BACKWARD = [(148, 1408), (149, 1408), (2048, 8), (2049, 8), (6000, 40), (2049, 264), (2500, 520), (3097, 1032), (1024, 8192), (1025, 8192), (3, 8200), (1, 8200)]


def _case(T, D, seed=0):
    r = np.random.default_rng([T, D, seed])
    bf = around.rne_bf16
    x, res = bf(r.normal(size=(T, D))), bf(r.normal(size=(T, D)) * 2.0 ** r.normal(size=(T, 1)))
    return x, res, bf(1 + 0.2 * r.normal(size=D)), bf(r.normal(size=(T, D))), bf(r.normal(size=(T, D)))


def _dev(a):
    return to_dev(f32_to_bf16(np.asarray(a, np.float32)).reshape(a.shape))


def _near(got, ref, tol):
    d = np.abs(f32(got).astype(np.float64) - ref)
    assert np.all(d <= tol), (float(np.max(d - tol)), np.argwhere(d > tol)[0])


def _codes_are_right(codes, scaled, extra):
    """Every code is within half a step of the value, the value's own float32 error allowed for."""
    v = f32(codes.view(torch.float8_e4m3fn)).astype(np.float64)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -20))), -6) - 3)
    d = np.abs(v - np.clip(scaled, -448, 448))
    assert np.all(d <= step / 2 * (1 + 2.0 ** -10) + extra * np.abs(scaled)), np.max(d / step)


@pytest.mark.parametrize("T,D", SHAPES)
def test_forward_and_backward(T, D):
    x, res, gamma, dY, dS = _case(T, D)
    eps = 1e-5
    S, r, y = around.rmsnorm_fwd(x, res, gamma, eps)
    X, R, G = _dev(x), _dev(res), _dev(gamma)
    out = {k: Guarded((T, D), BF) for k in ("sum", "Y", "dX")}
    rstd, dg, codes, scales = Guarded((T,), torch.float32), Guarded((D,), BF), Guarded((T, D)), Guarded((T,), torch.float32)
    ws = Guarded(b.sf_rmsnorm_bwd_workspace_size(T, D))
    got = b.sf_rmsnorm_fwd(X, G, eps, residual=R, sum=out["sum"].t, Y=out["Y"].t, codes=codes.t, scales=scales.t, rstd=rstd.t)
    assert got is out["Y"].t
    assert np.array_equal(f32(out["sum"].t), S)
    _near(out["Y"].t, y, (U16 + F32E) * np.abs(y))
    assert np.allclose(rstd.t.cpu().numpy(), r[:, 0], rtol=F32E)
    top = np.max(np.abs(y), axis=1)
    assert np.allclose(scales.t.cpu().numpy(), top / 448, rtol=F32E)
    _codes_are_right(codes.t, y / (top / 448)[:, None], 4 * F32E)
    # gradients, from the stored sum and the stored 1 / rms
    rd = rstd.t.cpu().numpy().astype(np.float64)[:, None]
    dX, dgamma = around.rmsnorm_bwd(dY, S, rd, gamma, dS)
    n, q = S * rd, dY * gamma
    b.sf_rmsnorm_bwd(_dev(dY), out["sum"].t, G, rstd.t, dS=_dev(dS), dX=out["dX"].t, dgamma=dg.t, workspace=ws.t)
    # dX: a mean of D products of four factors, and sums of three terms
    size = np.abs(dS) + rd * (np.abs(q) + np.abs(n) * np.mean(np.abs(q * n), axis=1, keepdims=True))
    _near(out["dX"].t, dX, U16 * np.abs(dX) + 2 * F32E * size)
    # dgamma: T products, added up over at most 296 CTAs of rows in turn
    _near(dg.t, dgamma, U16 * np.abs(dgamma) + (T / 296 + 64) * 2.0 ** -23 * np.sum(np.abs(dY * n), axis=0))
    again_x, again_g = b.sf_rmsnorm_bwd(_dev(dY), out["sum"].t, G, rstd.t, dS=_dev(dS))
    assert torch.equal(again_x, out["dX"].t) and torch.equal(again_g, dg.t)
    for g in [*out.values(), rstd, dg, codes, scales, ws]:
        g.check()


@pytest.mark.parametrize("T,D", BACKWARD)
def test_backward_of_short_and_long_batches(T, D):
    _, S, gamma, dY, dS = _case(T, D, 6)
    rstd = np.random.default_rng(T).uniform(0.1, 3, size=(T, 1)).astype(np.float32).astype(np.float64)
    dX, dgamma = around.rmsnorm_bwd(dY, S, rstd, gamma, dS)
    sd, G, r, dx, dg = _dev(S), _dev(gamma), torch.from_numpy(rstd[:, 0].astype(np.float32)).cuda(), Guarded((T, D), BF), Guarded((D,), BF)
    b.sf_rmsnorm_bwd(_dev(dY), sd, G, r, dS=_dev(dS), dX=dx.t, dgamma=dg.t)
    # bounds as above
    n, q = S * rstd, dY * gamma
    size = np.abs(dS) + rstd * (np.abs(q) + np.abs(n) * np.mean(np.abs(q * n), axis=1, keepdims=True))
    _near(dx.t, dX, U16 * np.abs(dX) + 2 * F32E * size)
    _near(dg.t, dgamma, U16 * np.abs(dgamma) + (T / 296 + 64) * 2.0 ** -23 * np.sum(np.abs(dY * n), axis=0))
    # one of the two alone, and in place: the same bits
    alone = b.sf_rmsnorm_bwd(_dev(dY), sd, G, r, dS=_dev(dS), dX=torch.empty_like(sd))[0]
    dgs = b.sf_rmsnorm_bwd(_dev(dY), sd, G, r, dgamma=torch.empty_like(G))[1]
    place = _dev(dY)
    both = b.sf_rmsnorm_bwd(place, sd, G, r, dS=_dev(dS), dX=place, dgamma=torch.empty_like(G))[1]
    assert torch.equal(alone, dx.t) and torch.equal(place, dx.t) and torch.equal(dgs, dg.t) and torch.equal(both, dg.t)
    dx.check()
    dg.check()


@pytest.mark.parametrize("T,D", [(3, 264), (200, 1408)])
def test_what_is_left_out(T, D):
    x, res, gamma, dY, dS = _case(T, D, 1)
    S, r, y = around.rmsnorm_fwd(x, None, gamma, 0.0)
    X, G = _dev(x), _dev(gamma)
    got = b.sf_rmsnorm_fwd(X, G, 0.0)
    _near(got, y, (U16 + F32E) * np.abs(y))
    codes = torch.zeros((T, D), dtype=torch.uint8, device="cuda")
    assert b.sf_rmsnorm_fwd(X, G, 0.0, codes=codes, scale=37.0) is codes
    _codes_are_right(codes, y * 37.0, 2 * F32E)
    rstd = torch.from_numpy(r[:, 0].astype(np.float32)).cuda()
    dX, dg = b.sf_rmsnorm_bwd(_dev(dY), X, G, rstd)
    want, want_g = around.rmsnorm_bwd(dY, S, r, gamma)
    assert np.linalg.norm(f32(dX) - want) < U16 * np.linalg.norm(want) and np.linalg.norm(f32(dg) - want_g) < U16 * np.linalg.norm(want_g)
    only = torch.zeros_like(X)
    assert b.sf_rmsnorm_bwd(_dev(dY), X, G, rstd, dX=only)[1] is None and torch.equal(only, dX)
    only = torch.zeros_like(G)
    assert b.sf_rmsnorm_bwd(_dev(dY), X, G, rstd, dgamma=only)[0] is None and torch.equal(only, dg)
    # the gradient in the place of either of the two that it is made of
    first = b.sf_rmsnorm_bwd(_dev(dY), X, G, rstd, dS=_dev(dS))[0]
    for name in ("dY", "dS"):
        t = {"dY": _dev(dY), "dS": _dev(dS)}
        b.sf_rmsnorm_bwd(t["dY"], X, G, rstd, dS=t["dS"], dX=t[name])
        assert torch.equal(t[name], first), name


def test_sum_in_place_and_strided_rows():
    T, D = 37, 1032
    x, res, gamma, _, _ = _case(T, D, 2)
    S, _, y = around.rmsnorm_fwd(x, res, gamma, 1e-6)
    wide = torch.full((T, D + 24), 7.0, dtype=BF, device="cuda")
    wide[:, :D] = _dev(x)
    R, G = _dev(res), _dev(gamma)
    Y = b.sf_rmsnorm_fwd(wide[:, :D], G, 1e-6, residual=R, sum=R)
    assert np.array_equal(f32(R), S) and bool((wide[:, D:] == 7).all())
    _near(Y, y, (U16 + F32E) * np.abs(y))
    X = _dev(x)
    assert torch.equal(b.sf_rmsnorm_fwd(X, G, 1e-6, residual=_dev(res), sum=X), Y) and np.array_equal(f32(X), S)
    big = torch.zeros((T + 3, D), dtype=BF, device="cuda")            # rows behind the last one are left as they were
    b.sf_rmsnorm_fwd(_dev(x), G, 1e-6, residual=_dev(res), Y=big[:T])
    assert torch.equal(big[:T], Y) and not big[T:].any()


def test_what_is_not_finite_or_zero():
    D = 520
    x = np.tile(around.rne_bf16(np.random.default_rng(5).normal(size=D)), (6, 1))
    x[1, 3], x[2, 4], x[3], x[4] = np.nan, np.inf, 0.0, x[4] * 2.0 ** -100
    x[5] *= 2.0 ** 40
    X, G = _dev(x), torch.ones(D, dtype=BF, device="cuda")
    codes, scales = torch.zeros((6, D), dtype=torch.uint8, device="cuda"), torch.zeros(6, device="cuda")
    Y = b.sf_rmsnorm_fwd(X, G, 1e-6, Y=torch.zeros_like(X), codes=codes, scales=scales)
    y, v = f32(Y), f32(codes.view(torch.float8_e4m3fn))
    assert np.isfinite(y[0]).all() and np.isnan(y[1]).all() and np.isnan(v[1]).all()
    assert np.isnan(y[2, 4]) and not np.delete(y[2], 4).any()
    assert not y[3].any() and not v[3].any() and scales[3] > 0
    assert np.abs(y[4]).max() < 1e-20 and np.isfinite(v[4]).all() and np.allclose(np.mean(y[5].astype(np.float64) ** 2), 1, rtol=1e-2)
    assert not f32(b.sf_rmsnorm_fwd(X[3:4], G, 1e-6)).any()
    assert np.isnan(f32(b.sf_rmsnorm_fwd(X[3:4], G, 0.0))).all()       # 0 / 0
    assert bool(torch.isnan(scales[1:3]).all()) and np.isnan(v[1:3]).all() and bool(torch.isfinite(scales[3:]).all())


def test_no_tokens():
    G = torch.ones(64, dtype=BF, device="cuda")
    X = torch.zeros((0, 64), dtype=BF, device="cuda")
    assert b.sf_rmsnorm_fwd(X, G, 1e-6).shape == (0, 64)
    dg = torch.ones_like(G)
    b.sf_rmsnorm_bwd(X, X, G, torch.zeros(0, device="cuda"), dX=torch.zeros_like(X), dgamma=dg)
    assert not dg.any()


def test_rows_beyond_32_bit_offsets():
    T, D = 131200, 32768
    X = torch.zeros((T, D), dtype=BF, device="cuda")
    X[-1] = _dev(_case(1, D, 3)[0])[0]
    X[0] = X[-1]
    G = torch.ones(D, dtype=BF, device="cuda")
    rstd = torch.empty(T, device="cuda")
    Y = b.sf_rmsnorm_fwd(X, G, 1e-6, Y=torch.empty_like(X), rstd=rstd)
    assert torch.equal(Y[0], Y[-1]) and bool(Y[0].any()) and not Y[1].any() and torch.equal(Y[-1], b.sf_rmsnorm_fwd(X[-1:], G, 1e-6)[0])
    dX = b.sf_rmsnorm_bwd(Y, X, G, rstd, dX=Y)[0]
    assert torch.equal(dX[0], dX[-1]) and bool(dX[0].any()) and not dX[1].any()


def test_captured_replayed_and_on_another_stream():
    T, D = 260, 512
    x, res, gamma, dY, dS = _case(T, D, 4)
    X, R, G, dy, ds = map(_dev, (x, res, gamma, dY, dS))
    S, Y, rstd, dX, dg = torch.empty_like(X), torch.empty_like(X), torch.empty(T, device="cuda"), torch.empty_like(X), torch.empty_like(G)
    ws = torch.empty(b.sf_rmsnorm_bwd_workspace_size(T, D), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        b.sf_rmsnorm_fwd(X, G, 1e-6, residual=R, sum=S, Y=Y, rstd=rstd, stream=stream)
        b.sf_rmsnorm_bwd(dy, S, G, rstd, dS=ds, dX=dX, dgamma=dg, workspace=ws, stream=stream)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (S, Y, dX, dg)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for t in (S, Y, dX, dg):
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    s.synchronize()
    assert all(torch.equal(a, w) for a, w in zip((S, Y, dX, dg), want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in (S, Y, dX, dg):
        t.zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for a, w in zip((S, Y, dX, dg), want))
