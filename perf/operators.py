"""The gated feed-forward block and the microscaled 4-bit operands of this package, as timed cases.

A case is one pass through one operator: the gated block forward, a training step of it (forward and backward), 4-bit
quantisation with its read-back, the product of two 4-bit operands, and the gated projection on such operands.
``run`` computes it with elementary torch operations, or (``own``) with the calls of
``paper_2602_06183_b200.binding``; ``exact`` computes it in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

BF16 = torch.bfloat16
# cost of the largest listed training step, in units of tokens x d_model x d_ffn; a drawn case costs no more
MAX_BLOCK = 8192 * 4096 * 16384
MAX_WEIGHT = 4096 * 16384
ACTS = ("silu", "gelu", "gelu_tanh", "relu", "sqrelu")


def listed():
    return [
        # One token of a decoding loop through the d_model 4096 layer: the three weight matrices are read once.
        {"name": "gated_token", "kind": "fwd", "T": 1, "D": 4096, "F": 16384, "act": "silu"},
        # A running batch of odd size through a layer whose sizes are no powers of two.
        {"name": "gated_batch_ragged", "kind": "fwd", "T": 77, "D": 1408, "F": 5504, "act": "gelu_tanh"},
        # A long prompt, nothing kept for a backward pass.
        {"name": "gated_prompt", "kind": "fwd", "T": 8192, "D": 4096, "F": 16384, "act": "silu"},
        # Training step of the parity-size layer: launches and latency are all of it.
        {"name": "gated_step_small", "kind": "step", "T": 256, "D": 256, "F": 1024, "act": "silu"},
        # Training step on an odd number of tokens, sizes that end inside every tile.
        {"name": "gated_step_ragged", "kind": "step", "T": 1999, "D": 1408, "F": 5504, "act": "gelu"},
        # Training step of the d_model 4096 layer.
        {"name": "gated_step_d4096", "kind": "step", "T": 8192, "D": 4096, "F": 16384, "act": "silu"},
        # The activation of one token on its way into a 4-bit product.
        {"name": "quant_token", "kind": "quant", "rows": 1, "cols": 4096, "fmt": "nv", "log2_scale": 3},
        # A weight matrix, blocks of 32 with power-of-two scales.
        {"name": "quant_weight", "kind": "quant", "rows": 16384, "cols": 4096, "fmt": "mx", "log2_scale": 0},
        # One token against a 4-bit weight matrix.
        {"name": "fp4_token", "kind": "gemm", "M": 1, "N": 16384, "K": 4096, "fmt": "nv"},
        # The shape of the E4M3 product sweep, its tokens as rows, blocks of 32.
        {"name": "fp4_product", "kind": "gemm", "M": 16384, "N": 4096, "K": 4096, "fmt": "mx"},
        # A handful of tokens through both projections on 4-bit weights.
        {"name": "fp4_gated_batch", "kind": "gated", "M": 5, "N": 16384, "K": 4096, "fmt": "nv", "act": "silu"},
        # An odd prompt through both projections.
        {"name": "fp4_gated_prompt", "kind": "gated", "M": 4099, "N": 8192, "K": 2048, "fmt": "nv", "act": "gelu_tanh"},
    ]


def _size(rng, lo, hi, multiple):
    """A multiple of `multiple` between lo and hi, even over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // multiple), min(hi // multiple, round(v / multiple))) * multiple


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "step", "step", "quant", "gemm", "gemm", "gated"])
    if kind == "quant":
        return {"kind": kind, "rows": _size(rng, 1, 16384, 1), "cols": _size(rng, 256, 4096, 32), "fmt": rng.choice(["nv", "mx"]),
                "log2_scale": rng.choice([-2, 0, 3])}
    while True:
        T, D, F = _size(rng, 1, 8192, 1), _size(rng, 256, 8192, 8), _size(rng, 256, 28672, 8)
        if T * D * F > MAX_BLOCK or D * F > MAX_WEIGHT:
            continue
        if kind in ("fwd", "step"):
            return {"kind": kind, "T": T, "D": D, "F": F, "act": rng.choice(ACTS)}
        case = {"kind": kind, "M": T, "N": F, "K": _size(rng, 256, 8192, 32), "fmt": rng.choice(["nv", "mx"])}
        if T * case["N"] * case["K"] > MAX_BLOCK or case["N"] * case["K"] > MAX_WEIGHT:
            continue
        if kind == "gated":
            case["act"] = rng.choice(ACTS)
        return case


def _normal(shape, std, gen):
    t = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    return t.mul_(std).to(BF16)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case)
    if case["kind"] in ("fwd", "step"):
        T, D, F = case["T"], case["D"], case["F"]
        s["X"] = _normal((T, D), 1.0, g)
        s["Wg"], s["Wu"] = _normal((F, D), 0.02, g), _normal((F, D), 0.02, g)
        s["Wd"] = _normal((D, F), 0.02, g)
        if case["kind"] == "step":
            s["dY"] = _normal((T, D), 1.0, g)
        return s
    if case["kind"] == "quant":
        # rows of different size, as activations and weight rows are
        r = torch.exp2(torch.randn((case["rows"], 1), generator=g, device="cuda"))
        s["X"] = (torch.randn((case["rows"], case["cols"]), generator=g, device="cuda") * r).to(BF16)
        return s
    # operands as a program holds them: codes, and scales in their tiles
    M, N, K, fmt = case["M"], case["N"], case["K"], case["fmt"]
    s["A"], s["As"] = _quantized(_normal((M, K), 1.0, g), fmt, 4.0)
    s["alpha"] = 1.0 / (4.0 * 512.0)
    s["B"], s["Bs"] = _quantized(_normal((N, K), 0.02, g), fmt, 512.0)
    if case["kind"] == "gated":
        s["B2"], s["B2s"] = _quantized(_normal((N, K), 0.02, g), fmt, 512.0)
    return s


# ---- the formats, in elementary operations ------------------------------------------------------------------
# E2M1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; a value half way between two goes to the one with the even code.


def _block(fmt):
    return 16 if fmt == "nv" else 32


def _e2m1(y):
    """Codes of y (any float type)."""
    a = y.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return c + 8 * torch.signbit(y).to(torch.uint8)


def _codes(x, fmt, scale):
    """bf16 [rows, cols] -> codes uint8 [rows, cols] and scale bytes uint8 [rows, cols / block]."""
    b = _block(fmt)
    v = (x.float() * scale).view(x.shape[0], -1, b)
    amax = v.abs().amax(dim=2)
    if fmt == "nv":
        sf = torch.clamp(amax / torch.full_like(amax, 6.0), max=448.0).to(torch.float8_e4m3fn)
        by, sf = sf.view(torch.uint8), sf.float()
    else:
        by = torch.clamp((amax.view(torch.int32) >> 23) - 2, min=0).to(torch.uint8)
        sf = torch.exp2(by.float() - 127.0)
    sf = sf.unsqueeze(2)
    y = torch.where(sf > 0, v / sf, torch.zeros_like(v))
    return _e2m1(y).view(x.shape), by


def _packed(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).contiguous()


def _tiled(by):
    """Scale bytes [rows, n] -> tiles of 128 rows x 4 scales, 512 bytes each: row r, scale c at 16 (r % 32) + 4 (r / 32) + c."""
    rows, n = by.shape
    R, C = -(-rows // 128), -(-n // 4)
    full = torch.zeros((R * 128, C * 4), dtype=torch.uint8, device=by.device)
    full[:rows, :n] = by
    return full.view(R, 4, 32, C, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _untiled(tiles, rows, n):
    R, C = -(-rows // 128), -(-n // 4)
    return tiles.view(R, C, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(R * 128, C * 4)[:rows, :n]


def _quantized(x, fmt, scale):
    c, by = _codes(x, fmt, scale)
    return _packed(c), _tiled(by)


def _scale_values(by, fmt, dtype):
    return by.contiguous().view(torch.float8_e4m3fn).to(dtype) if fmt == "nv" else torch.exp2(by.to(dtype) - 127)


def _values(packed, tiles, fmt, dtype):
    """What an operand stands for, before the scale of the whole tensor."""
    rows, K = packed.shape[0], 2 * packed.shape[1]
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=dtype, device=packed.device)
    v = table[torch.stack((packed & 15, packed >> 4), dim=2).view(rows, K).int()]
    sf = _scale_values(_untiled(tiles, rows, K // _block(fmt)), fmt, dtype)
    return (v.view(rows, -1, _block(fmt)) * sf.unsqueeze(2)).view(rows, K)


# ---- activations: value and derivative ------------------------------------------------------------------------


def _act(name, g):
    if name == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if name == "gelu":
        phi = 0.5 * torch.special.erfc(-g * math.sqrt(0.5))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * math.sqrt(0.5 / math.pi)
    if name == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = 1 / (1 + torch.exp(-c * (g + 0.044715 * g * g * g)))
        return g * s, s + g * s * (1 - s) * c * (1 + 3 * 0.044715 * g * g)
    r = torch.clamp(g, min=0)
    return (r, (g > 0).to(g.dtype)) if name == "relu" else (r * r, 2 * r)


def run(s):
    if own:
        return _run_own(s)
    kind = s["kind"]
    if kind == "quant":
        scale = 2.0 ** s["log2_scale"]
        c, by = _codes(s["X"], s["fmt"], scale)
        return {"Y": (_values(_packed(c), _tiled(by), s["fmt"], torch.float32) / scale).to(BF16)}
    if kind == "gemm":
        return {"C": (s["alpha"] * (_values(s["A"], s["As"], s["fmt"], torch.float32) @ _values(s["B"], s["Bs"], s["fmt"], torch.float32).T)).to(BF16)}
    if kind == "gated":
        a = _values(s["A"], s["As"], s["fmt"], torch.float32)
        g = s["alpha"] * (a @ _values(s["B"], s["Bs"], s["fmt"], torch.float32).T)
        u = s["alpha"] * (a @ _values(s["B2"], s["B2s"], s["fmt"], torch.float32).T)
        return {"H": (_act(s["act"], g)[0] * u).to(BF16)}
    x, wg, wu, wd = (s[k].float() for k in ("X", "Wg", "Wu", "Wd"))
    g, u = x @ wg.T, x @ wu.T
    a, da = _act(s["act"], g)
    h = a * u
    y = (h @ wd.T).to(BF16)
    if kind == "fwd":
        return {"Y": y}
    dy = s["dY"].float()
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    return {"Y": y, "dX": (dg @ wg + du @ wu).to(BF16), "dWg": (dg.T @ x).to(BF16), "dWu": (du.T @ x).to(BF16), "dWd": (dy.T @ h).to(BF16)}


def _run_own(s):
    from paper_2602_06183_b200 import binding
    kind = s["kind"]
    fmt = {"nv": binding.SF_FP4_NV, "mx": binding.SF_FP4_MX}[s["fmt"]] if "fmt" in s else None
    act = getattr(binding, "SF_ACT_" + s["act"].upper()) if "act" in s else None
    if kind == "quant":
        scale = 2.0 ** s["log2_scale"]
        s["q"] = binding.sf_fp4_quantize(s["X"], fmt, scale, out=s.get("q"))
        s["Y"] = binding.sf_fp4_dequantize(*s["q"], fmt, 1.0 / scale, out=s.get("Y"))
        return {"Y": s["Y"]}
    if kind in ("gemm", "gated"):
        if "ws" not in s:           # the buffers that a program keeps from call to call
            s["C"] = torch.empty((s["M"], s["N"]), dtype=BF16, device="cuda")
            s["ws"] = torch.zeros((binding.sf_gemm_fp4_workspace_size(s["M"], s["N"], s["K"]),), dtype=torch.uint8, device="cuda")
        if kind == "gemm":
            return {"C": binding.sf_gemm_fp4(s["A"], s["As"], s["B"], s["Bs"], fmt, s["alpha"], C_out=s["C"], workspace=s["ws"])}
        return {"H": binding.sf_gemm_fp4_gated(s["A"], s["As"], s["B"], s["Bs"], s["B2"], s["B2s"], fmt, act, s["alpha"], s["alpha"],
                                               H_out=s["C"], workspace=s["ws"])}
    if "ws" not in s:
        s["desc"] = binding.make_gated_desc(s["T"], s["D"], s["F"], act)
        s["ctx"], s["ws"] = binding.alloc_gated_ffn_buffers(s["desc"], training=kind == "step")
        s["Y"] = torch.empty_like(s["X"])
        if kind == "step":
            s |= {"d" + k: torch.empty_like(s[k]) for k in ("X", "Wg", "Wu", "Wd")}
    binding.sf_gated_ffn_fwd(s["desc"], s["X"], s["Wg"], s["Wu"], s["Wd"], s["Y"], s["ctx"], s["ws"])
    if kind == "fwd":
        return {"Y": s["Y"]}
    binding.sf_gated_ffn_bwd(s["desc"], s["dY"], s["X"], s["Wg"], s["Wu"], s["Wd"], s["ctx"], s["dX"], s["dWg"], s["dWu"], s["dWd"], s["ws"])
    return {k: s[k] for k in ("Y", "dX", "dWg", "dWu", "dWd")}


def work(case):
    kind = case["kind"]
    if kind in ("fwd", "step"):
        T, D, F = case["T"], case["D"], case["F"]
        if kind == "fwd":
            return {"bytes": 2 * (2 * T * D + 3 * F * D), "flops": 6 * T * D * F}
        return {"bytes": 2 * (4 * T * D + 6 * F * D), "flops": 18 * T * D * F}
    per = 0.5 + 1 / _block(case["fmt"])
    if kind == "quant":
        return {"bytes": int(case["rows"] * case["cols"] * (4 + 2 * per)), "flops": 4 * case["rows"] * case["cols"]}
    M, N, K, n = case["M"], case["N"], case["K"], 1 + (kind == "gated")
    return {"bytes": int((M + n * N) * K * per) + 2 * M * N, "flops": 2 * n * M * N * K}


# ---- in 64 bits, from the definitions ---------------------------------------------------------------------------


def _act64(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * (1 + torch.erf(g / math.sqrt(2))) / 2
    if name == "gelu_tanh":
        return g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))) / 2
    return torch.where(g > 0, g if name == "relu" else g * g, torch.zeros_like(g))


def _operand64(packed, tiles, fmt):
    """Value by value: sign, exponent and mantissa bit of every code, times its block's scale."""
    rows, K = packed.shape[0], 2 * packed.shape[1]
    code = torch.empty((rows, K), dtype=torch.int32, device=packed.device)
    code[:, 0::2], code[:, 1::2] = (packed & 15).int(), (packed >> 4).int()
    e, m = (code >> 1) & 3, (code & 1).double()
    mag = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e.double() - 1))
    v = torch.where(code >= 8, -mag, mag)
    n = K // _block(fmt)
    r, c = torch.arange(rows, device=packed.device).view(-1, 1), torch.arange(n, device=packed.device).view(1, -1)
    at = ((r // 128) * (-(-n // 4)) + c // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + c % 4
    by = tiles[at].int()
    if fmt == "nv":
        ee, mm = by >> 3, (by & 7).double()
        sf = torch.where(ee == 0, mm * 2.0 ** -9, (1 + mm / 8) * torch.exp2(ee.double() - 7))
    else:
        sf = torch.exp2(by.double() - 127)
    return v * sf.repeat_interleave(_block(fmt), dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quant":
        scale, b = 2.0 ** case["log2_scale"], _block(case["fmt"])
        x = (s["X"].double() * scale).view(case["rows"], -1, b)
        amax = x.abs().amax(dim=2, keepdim=True)
        if case["fmt"] == "nv":
            q = torch.clamp(amax / 6, max=448.0)
            step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(q, min=2.0 ** -20))), min=-6) - 3)
            sf = torch.round(q / step) * step           # three mantissa bits, ties to even
        else:
            sf = torch.exp2(torch.clamp(torch.frexp(amax).exponent.double() - 3, min=-127))
        y = torch.where(sf > 0, x / torch.where(sf > 0, sf, 1.0), 0.0)
        a = torch.clamp(y.abs(), max=6.0)
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        return {"Y": (torch.sign(y) * torch.round(a / step) * step * sf / scale).view(case["rows"], case["cols"])}
    if kind in ("gemm", "gated"):
        a = _operand64(s["A"], s["As"], case["fmt"])
        c = s["alpha"] * (a @ _operand64(s["B"], s["Bs"], case["fmt"]).T)
        if kind == "gemm":
            return {"C": c}
        return {"H": _act64(case["act"], c) * (s["alpha"] * (a @ _operand64(s["B2"], s["B2s"], case["fmt"]).T))}
    leaves = {k: s[k].double().requires_grad_(kind == "step") for k in ("X", "Wg", "Wu", "Wd")}
    h = _act64(case["act"], leaves["X"] @ leaves["Wg"].T) * (leaves["X"] @ leaves["Wu"].T)
    y = h @ leaves["Wd"].T
    if kind == "fwd":
        return {"Y": y}
    grads = torch.autograd.grad(y, list(leaves.values()), s["dY"].double())
    return {"Y": y.detach(), **{"d" + k: d for k, d in zip(leaves, grads)}}
