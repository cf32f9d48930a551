"""Microscaled 4-bit operands through the C ABI: the quantiser bit for bit on every bf16 pattern, its read-back, products that are exact
on small operands at every edge of the tiles, and the block trained in bf16 and served on 4 bits."""
import numpy as np
import pytest
import torch

from oracle import f32_to_bf16, fp4, gated
from paper_2602_06183_b200 import binding, synth
from util import Guarded, bits, f32, to_dev

pytestmark = pytest.mark.gpu

FMT = {"nv": binding.SF_FP4_NV, "mx": binding.SF_FP4_MX}


def _u8(t):
    return t.detach().contiguous().cpu().numpy()


def _dev8(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _check_quantized(got, x, fmt, scale):
    codes, by = fp4.quantize(x, fmt, scale)
    nan = np.repeat(np.isnan(fp4.scale_value(by, fmt)), fp4.BLOCK[fmt], axis=1)
    g = _u8(got[0])
    gc = np.empty_like(codes)
    gc[:, 0::2], gc[:, 1::2] = g & 15, g >> 4
    assert np.array_equal(gc[~nan], codes[~nan])               # a block whose scale is NaN has no defined codes
    off = fp4.tile_offsets(x.shape[0], -(-by.shape[1] // 4) * 4)
    padded = np.zeros(off.shape, np.uint8)
    padded[:, :by.shape[1]] = by
    assert np.array_equal(_u8(got[1])[off], padded)


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("scale", [1.0, 0.37, 64.0, 2.0 ** -9, 3.0e38])
def test_quantize_every_bf16_pattern(fmt, scale):
    r = np.random.default_rng(5)
    x = r.permutation(np.arange(65536, dtype=np.uint16)).reshape(256, 256)
    small = np.arange(65536, dtype=np.uint16).reshape(2048, 32)          # neighbours of one size: every ratio to the largest
    for v in (x, small):
        got = binding.sf_fp4_quantize(to_dev(v), FMT[fmt], scale)
        _check_quantized(got, v, fmt, scale)


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (1, 96), (3, 160), (31, 64), (33, 352), (127, 128), (129, 4096), (300, 992)])
def test_quantize_and_read_back(fmt, rows, cols):
    x = synth.normal_bf16((rows, cols), 0, 1, seed=rows + cols)
    x[rows // 2, :cols // 2] = 0                                          # blocks of zeros
    wide = torch.full((rows, cols + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :cols] = to_dev(x)
    n = binding.sf_fp4_sizes(rows, cols, FMT[fmt])
    codes, scales = Guarded((rows, cols // 2)), Guarded(n[1])
    scales.t.fill_(0x5A)
    binding.sf_fp4_quantize(wide[:, :cols], FMT[fmt], 4.0, out=(codes.t, scales.t))
    codes.check(); scales.check()   # noqa: E702
    _check_quantized((codes.t, scales.t), x, fmt, 4.0)
    # rows behind the last are left as they were
    used = fp4.tile_offsets(rows, -(-(cols // fp4.BLOCK[fmt]) // 4) * 4)
    rest = np.ones(n[1], bool)
    rest[used] = False
    assert (_u8(scales.t)[rest] == 0x5A).all()
    c, by = fp4.quantize(x, fmt, 4.0)
    want = fp4.values(c, by, fmt) / 4.0
    out = Guarded((rows, cols + 8), torch.bfloat16)
    out.t.fill_(5.0)
    binding.sf_fp4_dequantize(codes.t, scales.t, FMT[fmt], 0.25, out=out.t[:, :cols])
    out.check()
    assert np.array_equal(f32(out.t[:, :cols]).astype(np.float64), want)
    assert bool((out.t[:, cols:] == 5.0).all())


def _operand(rows, K, fmt, r, scales):
    """Random codes and scales, the tiles' unused rows full of NaN scales."""
    codes = r.integers(0, 16, size=(rows, K)).astype(np.uint8)
    by = r.choice(np.array(scales, np.uint8), size=(rows, K // fp4.BLOCK[fmt]))
    return fp4.values(codes, by, fmt), _dev8(fp4.pack(codes)), _dev8(fp4.tile(by, fill=0xFF if fmt == "mx" else 0x7F))


# powers of two from 1/2 to 2 (nv: E4M3 0x30, 0x38, 0x40): products are multiples of 1/16 below 144, sums of up to 7000 of them exact (below 2^20)
SIMPLE = {"nv": [0x30, 0x38, 0x40], "mx": [126, 127, 128]}
SHAPES = [(1, 8, 32), (1, 200, 96), (2, 128, 256), (5, 520, 1056), (16, 136, 288), (17, 264, 64), (33, 1032, 512), (64, 72, 800),
          (65, 392, 160), (128, 128, 1024), (129, 8, 32), (129, 264, 320), (200, 136, 544), (256, 256, 256), (257, 520, 1312), (520, 776, 96),
          (200, 136, 4096), (300, 1032, 4096), (513, 1032, 4096)]         # reductions split over four, three and two pairs


def _same(got, ref, what):
    g, r = bits(got), f32_to_bf16(ref.astype(np.float32)).reshape(ref.shape)
    bad = (g != r) & ~((g & 0x7FFF == 0) & (r & 0x7FFF == 0))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} differ, first at {tuple(np.argwhere(bad)[0])}"


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product_is_exact_on_simple_scales(fmt, M, N, K):
    r = np.random.default_rng(M + N + K)
    a, A, As = _operand(M, K, fmt, r, SIMPLE[fmt])
    b, B, Bs = _operand(N, K, fmt, r, SIMPLE[fmt])
    C, ws = Guarded((M, N), torch.bfloat16), Guarded(binding.sf_gemm_fp4_workspace_size(M, N, K), zero=True)
    binding.sf_gemm_fp4(A, As, B, Bs, FMT[fmt], 0.25, C_out=C.t, workspace=ws.t)
    assert binding.sf_check_status(ws.t) == binding.SF_OK
    C.check(); ws.check()   # noqa: E702
    _same(C.t, 0.25 * (a @ b.T), "C")
    if N % 8 == 0:
        g, Bg, Bgs = _operand(N, K, fmt, r, SIMPLE[fmt][:2])
        binding.sf_gemm_fp4_gated(A, As, Bg, Bgs, B, Bs, FMT[fmt], binding.SF_ACT_RELU, 0.5, 0.25, H_out=C.t, workspace=ws.t)
        assert binding.sf_check_status(ws.t) == binding.SF_OK
        C.check(); ws.check()   # noqa: E702
        G, U = 0.5 * (a @ g.T), 0.25 * (a @ b.T)
        # each factor is exact; their float32 product is one rounding, bf16's another
        H = (np.maximum(G, 0).astype(np.float32) * U.astype(np.float32)).astype(np.float64)
        _same(C.t, H, "H")


ALL_SCALES = {"nv": list(range(0x18, 0x58)), "mx": list(range(120, 134))}


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M,N,K", [(3, 264, 992), (100, 136, 512), (300, 392, 2080)])
def test_product_within_the_bounds(fmt, M, N, K):
    r = np.random.default_rng(K)
    a, A, As = _operand(M, K, fmt, r, ALL_SCALES[fmt])
    b, B, Bs = _operand(N, K, fmt, r, ALL_SCALES[fmt])
    alpha = 1 / 3
    C = binding.sf_gemm_fp4(A, As, B, Bs, FMT[fmt], alpha)
    ref, mag = alpha * (a @ b.T), alpha * (np.abs(a) @ np.abs(b).T)
    # K additions in float32, the product with alpha (itself a float32), the rounding to bf16
    tol = K * gated.ADD * mag + 2.0 ** -22 * np.abs(ref)
    tol = tol + gated.U16 * (np.abs(ref) + tol)
    assert np.all(np.abs(f32(C).astype(np.float64) - ref) <= tol)


@pytest.mark.parametrize("act", gated.ACTS)
@pytest.mark.parametrize("M", [4, 90, 300])
def test_gated_product_within_the_bounds(act, M):
    N, K, fmt = 200, 352, "nv"
    r = np.random.default_rng(M)
    a, A, As = _operand(M, K, fmt, r, ALL_SCALES[fmt])
    g, Bg, Bgs = _operand(N, K, fmt, r, ALL_SCALES[fmt])
    u, Bu, Bus = _operand(N, K, fmt, r, ALL_SCALES[fmt])
    ag = 2.0 ** -round(np.log2(np.std(a @ g.T)))
    H = binding.sf_gemm_fp4_gated(A, As, Bg, Bgs, Bu, Bus, FMT[fmt], binding.__dict__["SF_ACT_" + act.upper()], ag, ag)
    G, U = ag * (a @ g.T), ag * (a @ u.T)
    eg, eu = ag * K * gated.ADD * (np.abs(a) @ np.abs(g).T), ag * K * gated.ADD * (np.abs(a) @ np.abs(u).T)
    P, dP = gated.act(act, G)
    ep = (np.abs(dP) + 2 * eg) * eg + gated.ELEM * (1 + np.abs(G)) * np.abs(P)
    tol = (np.abs(P) + ep) * eu + np.abs(U) * ep
    tol = tol + gated.U16 * (np.abs(P * U) + tol)
    assert np.all(np.abs(f32(H).astype(np.float64) - P * U) <= tol)


@pytest.mark.parametrize("M", [6, 150])
def test_a_nan_block_reaches_its_row_only(M):
    N, K = 136, 320
    r = np.random.default_rng(2)
    x, w = synth.normal_bf16((M, K), 0, 1, seed=1), synth.normal_bf16((N, K), 0, 1, seed=2)
    B = binding.sf_fp4_quantize(to_dev(w), binding.SF_FP4_NV, 8.0)
    clean = f32(binding.sf_gemm_fp4(*binding.sf_fp4_quantize(to_dev(x), binding.SF_FP4_NV, 8.0), *B, binding.SF_FP4_NV, 1 / 64))
    x[3, r.integers(K)] = 0x7FC0
    C = f32(binding.sf_gemm_fp4(*binding.sf_fp4_quantize(to_dev(x), binding.SF_FP4_NV, 8.0), *B, binding.SF_FP4_NV, 1 / 64))
    rows = np.arange(M) != 3
    assert np.array_equal(C[rows], clean[rows]) and np.isnan(C[3]).all()


@pytest.mark.parametrize("M", [3, 200])
def test_captured_and_replayed(M):
    N, K = 264, 512
    x = [to_dev(synth.normal_bf16((M, K), 0, 1, seed=s)) for s in (1, 2)]
    B = binding.sf_fp4_quantize(to_dev(synth.normal_bf16((N, K), 0, 1, seed=3)), binding.SF_FP4_MX, 1.0)

    def chain(v, q, C, ws):
        binding.sf_fp4_quantize(v, binding.SF_FP4_MX, 2.0, out=q)
        binding.sf_gemm_fp4(*q, *B, binding.SF_FP4_MX, 0.5, C_out=C, workspace=ws)
    q = binding.sf_fp4_quantize(x[0], binding.SF_FP4_MX, 2.0)
    C, ws = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.zeros(256, dtype=torch.uint8, device="cuda")
    want = []
    for v in x:
        chain(v, q, C, ws)
        want.append(bits(C))
    buf = x[0].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        chain(buf, q, C, ws)
    for i in (1, 0, 1):
        buf.copy_(x[i])
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(bits(C), want[i])


def test_results_belong_to_the_stream_that_is_handed_over():
    """Memory that the current stream may still be using is not given to a call on another one."""
    M, N, K = 2048, 4096, 256
    A, B = (binding.sf_fp4_quantize(to_dev(synth.normal_bf16((n, K), 0, 1, seed=n)), binding.SF_FP4_NV, 1.0) for n in (M, N))
    want = bits(binding.sf_gemm_fp4(*A, *B, binding.SF_FP4_NV, 1.0))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()

    def freed(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda").data_ptr()
    at = freed(M, N)
    C = binding.sf_gemm_fp4(*A, *B, binding.SF_FP4_NV, 1.0, stream=s)
    s.synchronize()
    assert C.data_ptr() != at and np.array_equal(bits(C), want)
    at = freed(M, N)
    assert binding.sf_gemm_fp4_gated(*A, *B, *B, binding.SF_FP4_NV, 0, 1.0, 1.0, stream=s).data_ptr() != at
    at = freed(M, N // 2, dtype=torch.uint8)
    q = binding.sf_fp4_quantize(C, binding.SF_FP4_NV, 1.0, stream=s)
    assert q[0].data_ptr() != at
    at = freed(M, N)
    assert binding.sf_fp4_dequantize(*q, binding.SF_FP4_NV, 1.0, stream=s).data_ptr() != at
    s.synchronize()


@pytest.mark.parametrize("T", [1, 40, 300])
def test_trained_block_served_on_four_bits(T):
    """The two halves together, as they are used: a training step of the block in bf16, an update of its weights, the weights quantised
    once, and the block run on 4-bit operands: each stage against its own definition on the stage's own inputs."""
    D, F, fmt = 256, 512, "nv"
    r = np.random.default_rng(7)
    n = lambda s, k: to_dev(f32_to_bf16((r.normal(size=s) * k).astype(np.float32)).reshape(s))   # noqa: E731
    X, dY = n((T, D), 1.0), n((T, D), 1.0)
    W = {"Wg": n((F, D), 0.08), "Wu": n((F, D), 0.08), "Wd": n((D, F), 0.06)}
    desc = binding.make_gated_desc(T, D, F)
    ctx, ws = binding.alloc_gated_ffn_buffers(desc)
    Y, dX = torch.empty_like(X), torch.empty_like(X)
    grads = {k: torch.empty_like(v) for k, v in W.items()}
    binding.sf_gated_ffn_fwd(desc, X, W["Wg"], W["Wu"], W["Wd"], Y, ctx, ws)
    binding.sf_gated_ffn_bwd(desc, dY, X, W["Wg"], W["Wu"], W["Wd"], ctx, dX, grads["Wg"], grads["Wu"], grads["Wd"], ws)
    for k in W:
        assert bool(torch.isfinite(grads[k]).all())
        W[k] = W[k] - (1e-3 / max(1.0, T ** 0.5)) * grads[k]
    q = {k: binding.sf_fp4_quantize(v, FMT[fmt], 256.0) for k, v in W.items()}
    x = binding.sf_fp4_quantize(X, FMT[fmt], 64.0)
    H = binding.sf_gemm_fp4_gated(*x, *q["Wg"], *q["Wu"], FMT[fmt], binding.SF_ACT_SILU, 1 / (64 * 256), 1 / (64 * 256))
    h = binding.sf_fp4_quantize(H, FMT[fmt], 64.0)
    Y4 = binding.sf_gemm_fp4(*h, *q["Wd"], FMT[fmt], 1 / (64 * 256))
    assert binding.sf_check_status(ws) == binding.SF_OK

    def val(t, s):
        c, by = fp4.quantize(bits(t), fmt, s)
        return fp4.values(c, by, fmt) / s
    xv, gv, uv, dv = val(X, 64.0), val(W["Wg"], 256.0), val(W["Wu"], 256.0), val(W["Wd"], 256.0)
    P, dP = gated.act("silu", xv @ gv.T)
    U = xv @ uv.T
    e = D * gated.ADD * (np.abs(xv) @ np.abs(gv).T), D * gated.ADD * (np.abs(xv) @ np.abs(uv).T)
    tol = np.abs(P) * e[1] + np.abs(U) * (1.2 * e[0] + gated.ELEM * (1 + np.abs(xv @ gv.T)) * np.abs(P))
    tol = tol + gated.U16 * (np.abs(P * U) + tol)
    assert np.all(np.abs(f32(H).astype(np.float64) - P * U) <= tol)
    hv = val(H, 64.0)
    ref = hv @ dv.T
    tol = F * gated.ADD * (np.abs(hv) @ np.abs(dv).T)
    assert np.all(np.abs(f32(Y4).astype(np.float64) - ref) <= tol + gated.U16 * (np.abs(ref) + tol))




def test_offsets_beyond_32_bits():
    """A matrix of 4.4e9 elements: its last rows come out as a matrix of their own."""
    rows, cols, tail = 66_000, 66_560, 130
    X = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    X[-tail:] = torch.randn((tail, cols), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    last = rows - tail - (rows - tail) % 128                                # from the start of a tile of rows
    for fmt in (binding.SF_FP4_NV, binding.SF_FP4_MX):
        codes, scales = binding.sf_fp4_quantize(X, fmt, 2.0)
        c, s = binding.sf_fp4_quantize(X[last:], fmt, 2.0)
        assert torch.equal(codes[last:], c) and not bool(codes[:last].any())
        whole = s.numel() // 512 - (cols // (64 if fmt == binding.SF_FP4_NV else 128))         # tiles of whole row blocks of the tail
        assert torch.equal(scales[-s.numel():][:whole * 512], s[:whole * 512])
        back = binding.sf_fp4_dequantize(codes, scales, fmt, 0.5)
        assert torch.equal(back[last:], binding.sf_fp4_dequantize(c, s, fmt, 0.5)) and not bool(back[:last].any())
        del codes, scales, back
