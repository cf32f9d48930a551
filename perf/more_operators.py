"""What stands around the feed-forward layer in a step of training or serving, as timed cases.

A case is one pass through one operator: the root-mean-square norm that adds the residual (forward to bf16 and backward,
or forward to 8 bits with a scale to every token), the E4M3 product that takes such rows, the router's balance loss with its
gradients, and the orthogonalised update of a weight matrix. ``run`` computes it with elementary torch operations, or (``own``)
with the calls of ``paper_2602_06183_b200.binding``; ``exact`` computes it in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
ABC = (3.4445, -4.7750, 2.0315)         # the quintic of the Newton-Schulz iteration, as optimisers use it
# cost of the largest listed case of a kind; a drawn one costs no more
MAX_NORM = 16384 * 4096
MAX_PRODUCT = 8192 * 16384 * 4096
MAX_BALANCE = 16384 * 4096
MAX_ORTH = 4096 * 4096 * 16384


def listed():
    return [
        # One token of a decoding loop: residual stream in, operand of the layer out.
        {"name": "norm_token", "kind": "norm", "T": 1, "D": 4096, "eps": 1e-6},
        # One training batch of the d_model 4096 layer, forward and backward.
        {"name": "norm_step_d4096", "kind": "norm_step", "T": 16384, "D": 4096, "eps": 1e-6},
        # A ragged batch on a width that is no power of two.
        {"name": "norm_step_ragged", "kind": "norm_step", "T": 1999, "D": 1408, "eps": 1e-5},
        # A prompt on its way into an 8-bit product, a scale to every token.
        {"name": "norm_fp8_prompt", "kind": "norm_fp8", "T": 8192, "D": 4096, "eps": 1e-6},
        # A running batch of odd size, the same way.
        {"name": "norm_fp8_batch", "kind": "norm_fp8", "T": 77, "D": 8192, "eps": 1e-5},
        # One token against an 8-bit weight matrix.
        {"name": "fp8_token", "kind": "fp8", "M": 1, "N": 16384, "K": 4096},
        # The prompt's first product.
        {"name": "fp8_prompt", "kind": "fp8", "M": 8192, "N": 16384, "K": 4096},
        # A routed layer's batch: loss, counts, and the gradients of tokens and expert means.
        {"name": "balance_d4096", "kind": "balance", "T": 16384, "D": 4096, "E": 16},
        # A short ragged one with padded tokens.
        {"name": "balance_ragged", "kind": "balance", "T": 777, "D": 1408, "E": 5},
        # The update of a small layer's first matrix (more rows than columns), of sizes that end inside every tile.
        {"name": "orth_small", "kind": "orth", "rows": 1021, "cols": 253, "type": "f32"},
        # A middle-sized square one.
        {"name": "orth_square", "kind": "orth", "rows": 2048, "cols": 2048, "type": "bf16"},
        # The d_model 4096 layer's second matrix.
        {"name": "orth_d4096", "kind": "orth", "rows": 4096, "cols": 16384, "type": "bf16"},
    ]


def _size(rng, lo, hi, multiple=1):
    """A multiple of `multiple` between lo and hi, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // multiple), min(hi // multiple, round(v / multiple))) * multiple


def draw(rng):
    kind = rng.choice(["norm", "norm_step", "norm_step", "norm_fp8", "fp8", "fp8", "balance", "orth", "orth"])
    while True:
        if kind.startswith("norm"):
            c = {"kind": kind, "T": _size(rng, 1, 16384), "D": _size(rng, 64, 16384, 16 if kind == "norm_fp8" else 8), "eps": rng.choice([1e-6, 1e-5])}
            if c["T"] * c["D"] <= MAX_NORM:
                return c
        elif kind == "fp8":
            c = {"kind": kind, "M": _size(rng, 1, 8192), "N": _size(rng, 256, 16384, 8), "K": _size(rng, 256, 8192, 16)}
            if c["M"] * c["N"] * c["K"] <= MAX_PRODUCT and c["N"] * c["K"] <= 4096 * 16384:
                return c
        elif kind == "balance":
            c = {"kind": kind, "T": _size(rng, 1, 32768), "D": _size(rng, 128, 8192, 8), "E": rng.randint(1, 16)}
            if c["T"] * c["D"] <= MAX_BALANCE:
                return c
        else:
            c = {"kind": kind, "rows": _size(rng, 16, 16384), "cols": _size(rng, 16, 16384), "type": rng.choice(["bf16", "bf16", "f32"])}
            m, n = sorted((c["rows"], c["cols"]))
            if m * m * n <= MAX_ORTH and m * n <= 4096 * 16384:
                return c


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = dict(case)
    kind = case["kind"]
    if kind.startswith("norm"):
        T, D = case["T"], case["D"]
        # a residual stream whose tokens differ in size, and the layer output that is added to it
        s["R"] = (normal(T, D) * torch.exp2(normal(T, 1))).to(BF16)
        s["X"] = normal(T, D).to(BF16)
        s["gamma"] = (1 + 0.1 * normal(D)).to(BF16)
        if kind == "norm_step":
            s["dY"], s["dS"] = normal(T, D).to(BF16), normal(T, D).to(BF16)
    elif kind == "fp8":
        M, N, K = case["M"], case["N"], case["K"]
        x = normal(M, K) * torch.exp2(normal(M, 1))
        s["a_scales"] = (x.abs().amax(dim=1) / 448).contiguous()
        s["A"] = (x / s["a_scales"].unsqueeze(1)).to(E4M3).view(torch.uint8)
        s["B"] = (normal(N, K) * (0.02 * 2048)).clamp_(-448, 448).to(E4M3).view(torch.uint8)
        s["alpha"] = 1 / 2048
    elif kind == "balance":
        T, D, E = case["T"], case["D"], case["E"]
        s["X"] = normal(T, D).to(BF16)
        s["means"] = (normal(E, D) * (1.5 / math.sqrt(D))).to(BF16)
        s["logits"] = s["X"].float() @ s["means"].float().T
        s["expert"] = s["logits"].argmax(dim=1).to(torch.int32)
        if T > 16:
            s["expert"][T - T // 16:] = -1          # padding behind the last token
        # the layer's own gradient, of a mean over the tokens: about as large as what the loss adds to it
        s["dX_in"] = (normal(T, D) * (0.08 / T / math.sqrt(D))).to(BF16)
        s["cb"], s["cz"] = 0.01, 0.001
        s["dloss"] = torch.full((1,), 8.0, device="cuda")      # as a loss scale
    else:
        m, n = case["rows"], case["cols"]
        # an accumulated gradient: some directions carry most of it, the rest is spread over all
        r = min(m, n, 256)
        f = torch.arange(1, r + 1, device="cuda", dtype=F32) ** -0.5
        G = (normal(m, r) * f) @ normal(r, n) + 0.3 * normal(m, n)
        s["G"] = (G * 1e-3).to(BF16 if case["type"] == "bf16" else F32)
        s["steps"] = 5
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------


def _norm(s, dtype):
    """The sum as it is stored, 1 / rms of its rows, and the normalised rows in `dtype`."""
    S = (s["X"].float() + s["R"].float()).to(BF16)
    v = S.to(dtype)
    rstd = 1 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + s["eps"])
    return S, rstd, v * rstd


def run(s):
    if own:
        return _run_own(s)
    kind = s["kind"]
    if kind == "norm":
        S, _, n = _norm(s, F32)
        return {"sum": S, "Y": (n * s["gamma"].float()).to(BF16)}
    if kind == "norm_step":
        S, rstd, n = _norm(s, F32)
        dy = s["dY"].float()
        q = dy * s["gamma"].float()
        dx = s["dS"].float() + rstd * (q - n * (q * n).mean(dim=1, keepdim=True))
        return {"sum": S, "Y": (n * s["gamma"].float()).to(BF16), "dX": dx.to(BF16), "dgamma": (dy * n).sum(dim=0).to(BF16)}
    if kind == "norm_fp8":
        # in 64 bits: values next to a border between two codes
        S, _, n = _norm(s, torch.float64)
        y = n * s["gamma"].double()
        scale = y.abs().amax(dim=1, keepdim=True) / 448
        return {"sum": S, "codes": (y / scale).float().to(E4M3), "scales": scale.float().view(-1)}
    if kind == "fp8":
        a, b = s["A"].view(E4M3).float(), s["B"].view(E4M3).float()
        return {"C": (s["alpha"] * s["a_scales"].unsqueeze(1) * (a @ b.T)).to(BF16)}
    if kind == "balance":
        E, l = s["E"], s["logits"].double()            # in 64 bits: long sums
        here = s["expert"] >= 0
        counts = (s["expert"].unsqueeze(1) == torch.arange(E, device="cuda")).sum(dim=0)
        n = here.sum().double()
        top = l.amax(dim=1, keepdim=True)
        e = torch.exp(l - top)
        z = e.sum(dim=1, keepdim=True)
        p, lse = e / z, top + torch.log(z)
        w = here.unsqueeze(1).double()
        balance = E * (counts * (p * w).sum(dim=0)).sum() / (n * n)
        zloss = (lse * lse * w).sum() / n
        loss = torch.stack((s["cb"] * balance + s["cz"] * zloss, balance, zloss))
        c = counts.double()
        dl = w * s["dloss"].double() * p * (s["cb"] * E / (n * n) * (c - (p * c).sum(dim=1, keepdim=True)) + s["cz"] * 2 / n * lse)
        dl = dl.float()
        return {"loss": loss.float(), "counts": counts.to(torch.int32),
                "dX": (s["dX_in"].float() + dl @ s["means"].float()).to(BF16), "dmeans": (dl.T @ s["X"].float()).to(BF16)}
    a, b, c = ABC
    x = s["G"].float()
    wide = x.shape[0] <= x.shape[1]
    x = x if wide else x.T
    x = x / x.norm()
    x = _steps(x, s["steps"], a, b, c)
    return {"O": (x if wide else x.T).to(BF16).contiguous()}


def _steps(x, steps, a, b, c):
    if steps == 0:
        return x
    g = x @ x.T
    return _steps(a * x + (b * g + c * (g @ g)) @ x, steps - 1, a, b, c)


def _run_own(s):
    from paper_2602_06183_b200 import binding
    kind = s["kind"]
    if kind.startswith("norm"):
        if "S" not in s:            # the buffers that a program keeps from call to call
            T, D = s["T"], s["D"]
            s["S"], s["rstd"] = torch.empty_like(s["X"]), torch.empty((T,), dtype=F32, device="cuda")
            if kind == "norm_fp8":
                s["codes"], s["scales"] = torch.empty((T, D), dtype=torch.uint8, device="cuda"), torch.empty((T,), dtype=F32, device="cuda")
            else:
                s["Y"] = torch.empty_like(s["X"])
            if kind == "norm_step":
                s["dX"], s["dgamma"] = torch.empty_like(s["X"]), torch.empty_like(s["gamma"])
                s["ws"] = torch.empty((binding.sf_rmsnorm_bwd_workspace_size(T, D),), dtype=torch.uint8, device="cuda")
        if kind == "norm_fp8":
            binding.sf_rmsnorm_fwd(s["X"], s["gamma"], s["eps"], residual=s["R"], sum=s["S"], codes=s["codes"], scales=s["scales"])
            return {"sum": s["S"], "codes": s["codes"].view(E4M3), "scales": s["scales"]}
        binding.sf_rmsnorm_fwd(s["X"], s["gamma"], s["eps"], residual=s["R"], sum=s["S"], Y=s["Y"], rstd=s["rstd"] if kind == "norm_step" else None)
        if kind == "norm":
            return {"sum": s["S"], "Y": s["Y"]}
        binding.sf_rmsnorm_bwd(s["dY"], s["S"], s["gamma"], s["rstd"], dS=s["dS"], dX=s["dX"], dgamma=s["dgamma"], workspace=s["ws"])
        return {"sum": s["S"], "Y": s["Y"], "dX": s["dX"], "dgamma": s["dgamma"]}
    if kind == "fp8":
        if "ws" not in s:
            s["C"] = torch.empty((s["M"], s["N"]), dtype=BF16, device="cuda")
            s["ws"] = torch.zeros((binding.sf_gemm_fp8_rows_workspace_size(s["M"], s["N"], s["K"]),), dtype=torch.uint8, device="cuda")
        return {"C": binding.sf_gemm_fp8_rows(s["A"], s["a_scales"], s["B"], s["alpha"], C_out=s["C"], workspace=s["ws"])}
    if kind == "balance":
        if "ws" not in s:
            s["loss"], s["counts"] = torch.empty((3,), dtype=F32, device="cuda"), torch.empty((s["E"],), dtype=torch.int32, device="cuda")
            s["dX"], s["dmeans"] = torch.empty_like(s["X"]), torch.empty_like(s["means"])
            s["ws"] = torch.zeros((binding.sf_router_balance_workspace_size(s["T"], s["D"], s["E"]),), dtype=torch.uint8, device="cuda")
        binding.sf_router_balance_fwd(s["logits"], s["expert"], s["cb"], s["cz"], loss=s["loss"], counts=s["counts"], workspace=s["ws"])
        binding.sf_router_balance_bwd(s["logits"], s["expert"], s["counts"], s["cb"], s["cz"], s["X"], s["means"], dloss=s["dloss"], dX_in=s["dX_in"],
                                      dX=s["dX"], dmeans=s["dmeans"], workspace=s["ws"])
        return {k: s[k] for k in ("loss", "counts", "dX", "dmeans")}
    if "ws" not in s:
        s["O"] = torch.empty(s["G"].shape, dtype=BF16, device="cuda")
        s["ws"] = torch.zeros((binding.sf_orthogonalize_workspace_size(s["rows"], s["cols"]),), dtype=torch.uint8, device="cuda")
    return {"O": binding.sf_orthogonalize(s["G"], s["steps"], ABC, out=s["O"], workspace=s["ws"])}


def work(case):
    kind = case["kind"]
    if kind.startswith("norm"):
        T, D = case["T"], case["D"]
        if kind == "norm":
            return {"bytes": 8 * T * D + 2 * D, "flops": 6 * T * D}
        if kind == "norm_step":             # X, R, dY, dS in; sum, Y, dX out; the sum again where it no longer lies in a cache is not counted
            return {"bytes": 14 * T * D + 4 * D, "flops": 18 * T * D}
        return {"bytes": 7 * T * D + 2 * D + 4 * T, "flops": 8 * T * D}
    if kind == "fp8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + 2 * M * N + 4 * M, "flops": 2 * M * N * K}
    if kind == "balance":
        T, D, E = case["T"], case["D"], case["E"]
        return {"bytes": 6 * T * D + 4 * E * D + T * (4 * E + 4), "flops": 4 * T * D * E + 20 * T * E}
    m, n = sorted((case["rows"], case["cols"]))
    # both squares are symmetric: half of each is enough
    return {"bytes": m * n * (4 if case["type"] == "bf16" else 6), "flops": 5 * (3 * m * m * n + m ** 3)}


# ---- in 64 bits, from the definitions ---------------------------------------------------------------------------


def _e4m3_64(y):
    """The nearest value of E4M3 (three mantissa bits, ties to even, steps of 2^-9 at the bottom)."""
    e = torch.clamp(torch.frexp(y).exponent - 1, min=-6)
    step = torch.exp2(e.double() - 3)
    return torch.round(y / step) * step


def _e4m3_values(codes):
    c = codes.int()
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e.double() - 7))
    return torch.where(c >= 128, -v, v)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("norm"):
        S = (s["X"].double() + s["R"].double()).to(BF16).double()       # the sum is stored in bf16, and it is what is normalised
        leaf, gamma = S.clone().requires_grad_(True), s["gamma"].double().requires_grad_(True)
        y = leaf * torch.rsqrt(torch.mean(leaf ** 2, dim=1, keepdim=True) + case["eps"]) * gamma
        if kind == "norm":
            return {"sum": S, "Y": y.detach()}
        if kind == "norm_step":
            d, dg = torch.autograd.grad(y, (leaf, gamma), s["dY"].double())
            return {"sum": S, "Y": y.detach(), "dX": d + s["dS"].double(), "dgamma": dg}
        y = y.detach()
        scale = torch.max(torch.abs(y), dim=1).values / 448
        return {"sum": S, "codes": _e4m3_64(y / scale.unsqueeze(1)), "scales": scale}
    if kind == "fp8":
        return {"C": s["alpha"] * (s["a_scales"].double().unsqueeze(1) * _e4m3_values(s["A"])) @ _e4m3_values(s["B"]).T}
    if kind == "balance":
        T, E = case["T"], case["E"]
        keep = s["expert"] >= 0
        l = s["logits"].double().requires_grad_(True)
        counts = torch.bincount(s["expert"][keep].long(), minlength=E)
        k = l[keep]
        n = k.shape[0]
        balance = E * torch.sum(counts.double() / n * torch.softmax(k, dim=1).mean(dim=0))
        zloss = torch.mean(torch.logsumexp(k, dim=1) ** 2)
        total = s["cb"] * balance + s["cz"] * zloss
        dl, = torch.autograd.grad(total * s["dloss"].double()[0], l)
        return {"loss": torch.stack((total, balance, zloss)).detach(), "counts": counts.to(torch.int32),
                "dX": s["dX_in"].double() + dl @ s["means"].double(), "dmeans": dl.T @ s["X"].double()}
    # X_k = Q_k X_0 with Q_k a polynomial of the first square: all in the smaller of the two dimensions
    a, b, c = ABC
    G = s["G"].double()
    x = G if G.shape[0] <= G.shape[1] else G.T
    A = (x @ x.T) / torch.sum(x * x)
    eye = torch.eye(A.shape[0], dtype=torch.float64, device="cuda")
    Q = eye
    for _ in range(s["steps"]):
        B = a * eye + b * A + c * (A @ A)
        Q, A = B @ Q, B @ A @ B
    x = Q @ x / torch.sqrt(torch.sum(x * x))
    return {"O": x if G.shape[0] <= G.shape[1] else x.T.contiguous()}
