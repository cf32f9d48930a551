"""The norm, the layer, the balance loss and the update together, as a step uses them; each stage against the oracle on what the stage
before it left."""
import numpy as np
import pytest
import torch

from oracle import around, f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import f32, rel_fro, to_dev

pytestmark = pytest.mark.gpu
BF, E4, TOL = torch.bfloat16, torch.float8_e4m3fn, 2.0 ** -8


def _dev(a):
    return to_dev(f32_to_bf16(np.asarray(a, np.float32)).reshape(a.shape))


def _f64(t):
    return f32(t).astype(np.float64)


def test_training_step_of_a_routed_layer():
    T, D, F, E, eps, cb, cz = 512, 256, 1024, 4, 1e-5, 0.02, 0.001
    r = np.random.default_rng(9)
    bf = around.rne_bf16
    x, res, gamma = bf(r.normal(size=(T, D))), bf(r.normal(size=(T, D))), bf(1 + 0.1 * r.normal(size=D))
    X, R, G = _dev(x), _dev(res), _dev(gamma)
    W1, W2, means = _dev(r.normal(size=(F, D)) * 0.05), _dev(r.normal(size=(D, F)) * 0.05), _dev(r.normal(size=(E, D)) * 0.1)
    dOut = _dev(r.normal(size=(T, D)) / T)

    S, rstd, N = torch.empty_like(X), torch.empty(T, device="cuda"), torch.empty_like(X)
    b.sf_rmsnorm_fwd(X, G, eps, residual=R, sum=S, Y=N, rstd=rstd)
    d = b.make_router_desc(T, D, F, E)
    cbytes, wbytes = b.sf_routed_ffn_workspace_size(d)
    ctx, ws = torch.zeros(cbytes, dtype=torch.uint8, device="cuda"), torch.zeros(wbytes, dtype=torch.uint8, device="cuda")
    Y = torch.empty_like(X)
    b.sf_routed_ffn_fwd(d, N, W1, W2, means, Y, ctx, ws)
    expert = b.sf_routed_ctx_view(d, ctx, b.SF_RCTX_EXPERT).view(torch.int32)
    logits = b.sf_routed_ctx_view(d, ctx, b.SF_RCTX_LOGITS).view(torch.float32).view(T, E)
    loss, counts = b.sf_router_balance_fwd(logits, expert, cb, cz)

    # the step's result is S + Y: its gradient comes to S directly and through the layer
    dN, dW1, dW2 = torch.empty_like(N), torch.empty_like(W1), torch.empty_like(W2)
    b.sf_routed_ffn_bwd(d, dOut, N, W1, W2, ctx, dN, dW1, dW2, ws)
    layer = _f64(dN)
    dmeans = torch.empty_like(means)
    b.sf_router_balance_bwd(logits, expert, counts, cb, cz, N, means, dX_in=dN, dX=dN, dmeans=dmeans)
    dX, dgamma = b.sf_rmsnorm_bwd(dN, S, G, rstd, dS=dOut)
    updates = [b.sf_orthogonalize(w) for w in (dW1, dW2)]
    torch.cuda.synchronize()

    ref_S, ref_r, ref_N = around.rmsnorm_fwd(x, res, gamma, eps)
    assert np.array_equal(f32(S), ref_S) and rel_fro(f32(N), ref_N) < TOL
    lg, ex = logits.double().cpu().numpy(), expert.cpu().numpy()
    assert np.allclose(lg, _f64(N) @ _f64(means).T, atol=1e-4)
    want, n = around.balance_fwd(lg, ex, cb, cz)
    assert np.array_equal(counts.cpu().numpy(), n) and np.allclose(loss.cpu().numpy(), want, rtol=2.0 ** -16)
    want_dn, want_dm, _ = around.balance_bwd(lg, ex, cb, cz, _f64(N), _f64(means), 1.0, layer)
    assert rel_fro(_f64(dN), want_dn) < TOL and rel_fro(_f64(dmeans), want_dm) < TOL
    want_dx, want_dg = around.rmsnorm_bwd(_f64(dN), _f64(S), rstd.double().cpu().numpy()[:, None], gamma, _f64(dOut))
    assert rel_fro(_f64(dX), want_dx) < TOL and rel_fro(_f64(dgamma), want_dg) < TOL
    for u, w in zip(updates, (dW1, dW2)):
        e = around.orthogonalize(_f64(w))
        made = np.linalg.norm(around.orthogonalize_rounded(_f64(w)) - e) / np.linalg.norm(e)
        assert rel_fro(_f64(u), e) < TOL + 2 * made


@pytest.mark.parametrize("T", [1, 40, 300])
def test_serving_in_eight_bits(T):
    """Norm to 8-bit rows, and the product that takes them: within the roundings to E4M3 of what float64 makes of the same weights."""
    D, F = 512, 1032
    r = np.random.default_rng(T)
    bf = around.rne_bf16
    x, res, gamma, w = bf(r.normal(size=(T, D))), bf(r.normal(size=(T, D))), bf(1 + 0.1 * r.normal(size=D)), bf(r.normal(size=(F, D)) * 0.03)
    R = _dev(res)
    codes, scales = torch.empty((T, D), dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    b.sf_rmsnorm_fwd(_dev(x), _dev(gamma), 1e-6, residual=R, sum=R, codes=codes, scales=scales)
    Wq = b.sf_fp8_quantize(_dev(w), 2048.0)
    C = b.sf_gemm_fp8_rows(codes, scales, Wq, 1 / 2048)
    q, v = codes.view(E4).double().cpu().numpy() * scales.double().cpu().numpy()[:, None], Wq.view(E4).double().cpu().numpy() / 2048
    assert rel_fro(_f64(C), q @ v.T) < TOL                                     # the product itself
    y = around.rmsnorm_fwd(x, res, gamma, 1e-6)[2]
    # half a step of either operand, 2^-4 at most each; their errors are independent of one another and of the sums' signs
    assert rel_fro(_f64(C), y @ w.T) < 2 * 2.0 ** -4
