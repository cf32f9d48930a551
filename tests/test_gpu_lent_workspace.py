"""One buffer, zeroed once, lent to one call after the other: each leaves it so that the next finds what it needs (the status word at 0, and no trace
of itself in the first 256 bytes), and every result has the bits that a workspace of its own gives."""
import pytest
import torch

from paper_2602_06183_b200 import binding as b

pytestmark = pytest.mark.gpu
BF, U8 = torch.bfloat16, torch.uint8


def _normal(*shape):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(sum(shape)), device="cuda")


def norm(T, D):
    dY, S, G, r = _normal(T, D).to(BF), _normal(D, T).T.contiguous().to(BF), _normal(D).to(BF), _normal(T).abs()
    return b.sf_rmsnorm_bwd_workspace_size(T, D), lambda ws: b.sf_rmsnorm_bwd(dY, S, G, r, dX=torch.zeros_like(S), dgamma=torch.zeros_like(G), workspace=ws)


def balance(T, D, E):
    X, m = _normal(T, D).to(BF), (_normal(E, D) * 0.1).to(BF)
    L = X.float() @ m.float().T
    ex = L.argmax(1).int()

    def run(ws):
        loss, n = b.sf_router_balance_fwd(L, ex, 0.5, 0.1, workspace=ws)
        return loss, n, *b.sf_router_balance_bwd(L, ex, n, 0.5, 0.1, X, m, dX=torch.zeros_like(X), dmeans=torch.zeros_like(m), workspace=ws)
    return b.sf_router_balance_workspace_size(T, D, E), run


def rows(M, N, K):
    A, B = (_normal(n, K).to(torch.float8_e4m3fn).view(U8) for n in (M, N))
    s = _normal(M).abs()
    return b.sf_gemm_fp8_rows_workspace_size(M, N, K), lambda ws: (b.sf_gemm_fp8_rows(A, s, B, 0.5, workspace=ws),)


def update(m, n):
    G = _normal(m, n).to(BF)
    return b.sf_orthogonalize_workspace_size(m, n), lambda ws: (b.sf_orthogonalize(G, workspace=ws),)


def test_every_call_in_turn():
    calls = [make(*a) for make, a in ((norm, (2500, 520)), (balance, (5000, 136, 6)), (norm, (2049, 264)), (rows, (3, 264, 528)), (norm, (4100, 4104)),
                                      (balance, (40000, 24, 16)), (update, (200, 333)), (norm, (300, 8200)), (rows, (300, 264, 528)), (balance, (100, 64, 3)))]
    lent = torch.zeros(max(n for n, _ in calls), dtype=U8, device="cuda")
    for _ in range(2):
        for i, (n, run) in enumerate(calls):
            got = [t.clone() for t in run(lent)]
            assert b.sf_check_status(lent) == b.SF_OK, i
            assert not lent[:256].any(), i
            want = run(torch.zeros(n, dtype=U8, device="cuda"))
            assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(got, want)), i
