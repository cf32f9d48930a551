"""The router's balance loss and its gradients through the C ABI, against the oracle in 64 bits: every number of experts, padded tokens whose
rows hold anything, sharp and masked logits, ragged sizes, what is left out.

Bounds. The loss: float32 probabilities (exponential and quotient, a few 2^-23), sums of at most T / 37888 + 300 terms. dl: relative 2^-18
for a sum of two bf16 numbers (2^-17 with its own float32 arithmetic, whose difference n_e - sum n_j p_j is taken relative to n)."""
import numpy as np
import pytest
import torch

from oracle import around, f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import Guarded, f32, to_dev

pytestmark = pytest.mark.gpu
BF, U16 = torch.bfloat16, 2.0 ** -8


def _dev(a):
    return to_dev(f32_to_bf16(np.asarray(a, np.float32)).reshape(a.shape))


def _case(T, D, E, seed=0, pad=True):
    r = np.random.default_rng([T, D, E, seed])
    X, means = around.rne_bf16(r.normal(size=(T, D))), around.rne_bf16(r.normal(size=(E, D)) * 2 / np.sqrt(D))
    logits = (X @ means.T).astype(np.float32).astype(np.float64)
    expert = np.argmax(logits, axis=1).astype(np.int32)
    if pad and T > 4:
        expert[r.random(T) < 0.2] = -1
        expert[T // 2] = E
    return X, means, logits, expert, r


def _check(X, means, logits, expert, cb, cz, dX_in=None, dloss=None):
    (T, D), E = X.shape, means.shape[0]
    L, ex = torch.from_numpy(logits.astype(np.float32)).cuda(), torch.from_numpy(expert).cuda()
    loss, counts = Guarded((3,), torch.float32), Guarded((E,), torch.int32)
    dX, dm, ws = Guarded((T, D), BF), Guarded((E, D), BF), Guarded(b.sf_router_balance_workspace_size(T, D, E), zero=True)
    b.sf_router_balance_fwd(L, ex, cb, cz, loss=loss.t, counts=counts.t, workspace=ws.t)
    want, n = around.balance_fwd(logits, expert, cb, cz)
    assert np.array_equal(counts.t.cpu().numpy(), n)
    with np.errstate(over="ignore"):
        want = want.astype(np.float32)                     # the type of the result: what its range does not hold is infinite
    assert np.allclose(loss.t.cpu().numpy(), want, rtol=2.0 ** -17, atol=1e-30), (loss.t, want)
    g = None if dloss is None else torch.full((1,), dloss, device="cuda")
    b.sf_router_balance_bwd(L, ex, counts.t, cb, cz, _dev(X), _dev(means), dloss=g, dX_in=None if dX_in is None else _dev(dX_in), dX=dX.t, dmeans=dm.t,
                            workspace=ws.t)
    assert b.sf_check_status(ws.t) == b.SF_OK
    wx, wm, dl = around.balance_bwd(logits, expert, cb, cz, X, means, 1.0 if dloss is None else dloss, dX_in)
    # dl's own error, of the size of its largest part
    p, lse = around.softmax(logits)
    total = max(int(n.sum()), 1)
    here = (expert >= 0) & (expert < E)
    part = (abs(cb) * E / total ** 2 * (n[None] + (np.nan_to_num(p) @ n)[:, None]) + 2 * abs(cz) / total * np.abs(lse)[:, None]) * p * abs(1 if dloss is None else dloss)
    e = np.where(here[:, None], 2.0 ** -16 * part, 0)
    Xs = np.where(here[:, None], np.abs(X), 0)
    base = 0 if dX_in is None else np.abs(dX_in)
    tiny = 2.0 ** -130
    got = f32(dX.t).astype(np.float64)
    assert np.all(np.abs(got - wx) <= U16 * np.abs(wx) + e @ np.abs(means) + 2.0 ** -20 * (base + np.abs(dl) @ np.abs(means)) + tiny)
    got = f32(dm.t).astype(np.float64)
    assert np.all(np.abs(got - wm) <= U16 * np.abs(wm) + e.T @ Xs + (T / 148 + 200) * 2.0 ** -23 * (np.abs(dl).T @ Xs) + tiny)
    for x in (loss, counts, dX, dm, ws):
        x.check()
    return dX.t, dm.t


@pytest.mark.parametrize("E", list(range(1, 17)))
def test_every_number_of_experts(E):
    X, means, logits, expert, r = _case(300, 136, E)
    _check(X, means, logits, expert, 0.02, 0.003, dX_in=around.rne_bf16(r.normal(size=X.shape) * 1e-4), dloss=3.0)


@pytest.mark.parametrize("T,D", [(1, 8), (3, 1032), (31, 64), (32, 72), (33, 512), (255, 520), (257, 1408), (2000, 256), (5000, 4096), (40000, 24),
                                 # one launch up to eight tiles of 32 tokens and 64 CTAs, and two beyond
                                 (256, 520), (224, 1024), (256, 4096), (256, 4104), (160, 6144), (40, 16384), (2, 80000)])
def test_sizes(T, D):
    X, means, logits, expert, r = _case(T, D, 6)
    dX, dm = _check(X, means, logits, expert, 0.02, 0.003)
    L, ex = torch.from_numpy(logits.astype(np.float32)).cuda(), torch.from_numpy(expert).cuda()
    n = b.sf_router_balance_fwd(L, ex, 0.02, 0.003)[1]
    again = b.sf_router_balance_bwd(L, ex, n, 0.02, 0.003, _dev(X), _dev(means))
    assert torch.equal(again[0], dX) and torch.equal(again[1], dm)
    # one of the two alone; and dX in the place of what it is added to
    x, m = torch.zeros_like(dX), torch.zeros_like(dm)
    b.sf_router_balance_bwd(L, ex, n, 0.02, 0.003, _dev(X), _dev(means), dX=x)
    b.sf_router_balance_bwd(L, ex, n, 0.02, 0.003, _dev(X), _dev(means), dmeans=m)
    assert torch.equal(x, dX) and torch.equal(m, dm)
    add = _dev(around.rne_bf16(r.normal(size=X.shape) * 1e-3))
    want = b.sf_router_balance_bwd(L, ex, n, 0.02, 0.003, _dev(X), _dev(means), dX_in=add, dX=x)[0].clone()
    b.sf_router_balance_bwd(L, ex, n, 0.02, 0.003, _dev(X), _dev(means), dX_in=add, dX=add)
    assert torch.equal(add, want)


@pytest.mark.parametrize("E", [1, 2, 7, 13, 16])
def test_every_number_of_experts_of_a_short_batch(E):
    X, means, logits, expert, r = _case(200, 584, E)
    _check(X, means, logits, expert, 0.02, 0.003, dX_in=around.rne_bf16(r.normal(size=X.shape) * 1e-4), dloss=3.0)


def test_tokens_that_are_left_out_may_hold_anything():
    X, means, logits, expert, r = _case(500, 264, 7)
    out = (expert < 0) | (expert >= 7)
    clean = _check(X, means, logits, expert, 0.02, 0.003)
    X[out], logits[out] = np.nan, np.inf
    L, ex = torch.from_numpy(logits.astype(np.float32)).cuda(), torch.from_numpy(expert).cuda()
    loss, n = b.sf_router_balance_fwd(L, ex, 0.02, 0.003)
    assert bool(torch.isfinite(loss).all())
    got = b.sf_router_balance_bwd(L, ex, n, 0.02, 0.003, _dev(X), _dev(means))
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1]) and not got[0][torch.from_numpy(out).cuda()].any()


@pytest.mark.parametrize("T", [1, 700])
def test_no_token_counts(T):
    X, means, logits, _, _ = _case(T, 64, 3)
    _check(X, means, logits, np.full(T, -1, np.int32), 0.5, 0.5)
    _check(X, means, logits, np.full(T, 2 ** 31 - 1, np.int32), 0.5, 0.5, dX_in=X)


def test_sharp_masked_and_lowest_logits():
    X, means, logits, _, r = _case(400, 64, 5)
    logits = (logits * 1e3).astype(np.float32).astype(np.float64)
    logits[:100, 1] = -np.inf
    logits[100:200, 2] = np.float64(np.finfo(np.float32).min)
    logits[200:210] = np.float64(np.finfo(np.float32).min)
    expert = np.argmax(logits, axis=1).astype(np.int32)
    with np.errstate(over="ignore"):
        _check(X, means, logits, expert, 0.02, 0.0)
    logits[200:210] = 88.0
    _check(X, means, logits, expert, 0.02, 1e-6)


def test_everything_at_one_expert():
    X, means, logits, _, _ = _case(1000, 64, 16)
    _check(X, means, logits, np.full(1000, 15, np.int32), 1.0, 0.0)


def test_no_tokens():
    L, ex = torch.zeros((0, 4), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    loss, n = b.sf_router_balance_fwd(L, ex, 1.0, 1.0)
    assert not loss.any() and not n.any()
    X, m = torch.zeros((0, 64), dtype=BF, device="cuda"), torch.ones((4, 64), dtype=BF, device="cuda")
    dm = torch.ones_like(m)
    b.sf_router_balance_bwd(L, ex, n, 1.0, 1.0, X, m, dmeans=dm)
    assert not dm.any()


def test_follows_the_router():
    """On what sf_router_route writes."""
    X, means, _, _, _ = _case(512, 256, 8)
    ex, L = b.sf_router_route(_dev(X), _dev(means))
    loss, n = b.sf_router_balance_fwd(L, ex, 1.0)
    want, counts = around.balance_fwd(L.double().cpu().numpy(), ex.cpu().numpy(), 1.0, 0.0)
    assert np.array_equal(n.cpu().numpy(), counts) and np.allclose(loss.cpu().numpy(), want, rtol=2.0 ** -17)


def test_captured_twice_and_replayed():
    X, means, logits, expert, _ = _case(700, 264, 9)
    L, ex, x, m = torch.from_numpy(logits.astype(np.float32)).cuda(), torch.from_numpy(expert).cuda(), _dev(X), _dev(means)
    loss, n, dX, dm = torch.zeros(3, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda"), torch.zeros_like(x), torch.zeros_like(m)
    ws = torch.zeros(b.sf_router_balance_workspace_size(700, 264, 9), dtype=torch.uint8, device="cuda")

    def step():
        b.sf_router_balance_fwd(L, ex, 0.1, 0.2, loss=loss, counts=n, workspace=ws)
        b.sf_router_balance_bwd(L, ex, n, 0.1, 0.2, x, m, dX=dX, dmeans=dm, workspace=ws)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (loss, n, dX, dm)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
        step()
    for t in (loss, n, dX, dm):
        t.zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, w) for a, w in zip((loss, n, dX, dm), want))
