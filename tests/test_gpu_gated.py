"""The gated feed-forward block through the C ABI: exact on small integers at every edge of the tiles, within derived bounds for every
activation, captured and replayed, on another stream, and with everything around its buffers left alone."""
import numpy as np
import pytest
import torch

from oracle import f32_to_bf16, gated
from paper_2602_06183_b200 import binding
from util import Guarded, bits, f32, to_dev

pytestmark = pytest.mark.gpu

GRADS = ("dX", "dWg", "dWu", "dWd")


def _ints(shape, r, lo=-2, hi=2, keep=0.3):
    """Small integers, most of them zero: sums stay exact in float32."""
    return (r.integers(lo, hi + 1, size=shape) * (r.random(shape) < keep)).astype(np.float64)


def _dev(a):
    return to_dev(f32_to_bf16(a.astype(np.float32)).reshape(a.shape))


class Block:
    """A block's tensors on the device, every buffer between guards."""

    def __init__(self, T, D, F, act, X, Wg, Wu, Wd, dY=None, training=True):
        self.desc = binding.make_gated_desc(T, D, F, binding.__dict__["SF_ACT_" + act.upper()])
        c, w = binding.sf_gated_ffn_workspace_size(self.desc)
        self.ctx = Guarded(c) if training else None
        self.ws = Guarded(w)
        self.ws.t[:256].zero_()
        self.X, self.Wg, self.Wu, self.Wd = map(_dev, (X, Wg, Wu, Wd))
        self.Y = Guarded((T, D), torch.bfloat16)
        if dY is not None:
            self.dY = _dev(dY)
            self.out = {k: Guarded(tuple(getattr(self, k[1:]).shape), torch.bfloat16) for k in GRADS}

    def fwd(self, stream=None):
        binding.sf_gated_ffn_fwd(self.desc, self.X, self.Wg, self.Wu, self.Wd, self.Y.t, self.ctx.t if self.ctx else None, self.ws.t, stream=stream)

    def bwd(self, only=GRADS, stream=None):
        o = [self.out[k].t if k in only else None for k in GRADS]
        binding.sf_gated_ffn_bwd(self.desc, self.dY, self.X, self.Wg, self.Wu, self.Wd, self.ctx.t, *o, self.ws.t, stream=stream)

    def check(self):
        assert binding.sf_check_status(self.ws.t) == binding.SF_OK
        for g in [self.ctx, self.ws, self.Y, *getattr(self, "out", {}).values()]:
            if g is not None:
                g.check()


def _same(got, ref, what):
    g = bits(got)
    r = f32_to_bf16(ref.astype(np.float32)).reshape(ref.shape)
    bad = (g != r) & ~((g & 0x7FFF == 0) & (r & 0x7FFF == 0))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} differ, first at {tuple(np.argwhere(bad)[0])}"


def _within(got, ref, tol, what):
    d = np.abs(f32(got).astype(np.float64) - ref)
    assert np.all(d <= tol), f"{what}: {(d > tol).sum()} of {d.size} outside, worst {np.max(d / np.maximum(tol, 1e-300)):.3g} of the bound"


# one token to more than a tile of 256; D and F: one 16-byte unit, below and above a block of 64, odd multiples of 8, several tiles
SHAPES = [(1, 8, 8), (1, 264, 520), (2, 72, 136), (7, 1000, 328), (16, 64, 128), (17, 128, 64), (33, 520, 1032), (64, 256, 256),
          (65, 136, 392), (128, 200, 776), (129, 8, 16), (129, 264, 520), (200, 584, 72), (256, 256, 512), (257, 392, 1160), (513, 136, 264)]


# every product of the step in every form that it has beyond the few tokens above (see test_gated_plan.py): persistent tiles of full and
# of narrower width, and reductions split over two to four pairs
FORM_SHAPES = [(130, 1408, 8), (130, 8, 1032), (257, 392, 1160), (513, 256, 2048), (513, 520, 2048), (513, 776, 1160), (513, 2048, 520),
               (513, 1024, 1032), (513, 1408, 1032), (1000, 8, 8), (1500, 1032, 8), (1000, 4096, 520), (3000, 256, 2048),
               (3000, 1024, 1160), (4096, 776, 264), (1295, 1120, 2360), (65, 1096, 136), (128, 1032, 200)]


@pytest.mark.parametrize("T,D,F", SHAPES + FORM_SHAPES)
def test_step_is_exact_on_small_integers(T, D, F):
    r = np.random.default_rng(T * 7 + D + F)
    X, Wg, Wu, Wd, dY = _ints((T, D), r), _ints((F, D), r, -1, 1), _ints((F, D), r, -1, 1), _ints((D, F), r, -1, 1, 0.1), _ints((T, D), r, -1, 1)
    ref = gated.exact_step(X, Wg, Wu, Wd, dY)
    b = Block(T, D, F, "relu", X, Wg, Wu, Wd, dY)
    b.fwd()
    b.bwd()
    b.check()
    _same(b.Y.t, ref["Y"], "Y")
    for k in GRADS:
        _same(b.out[k].t, ref[k], k)
    # without a context: the same Y, bit for bit
    i = Block(T, D, F, "relu", X, Wg, Wu, Wd, training=False)
    i.fwd()
    i.check()
    assert np.array_equal(bits(i.Y.t), bits(b.Y.t))


def _normals(T, D, F, seed):
    r = np.random.default_rng(seed)
    def n(shape, s):
        return gated.rne_bf16(r.normal(size=shape) * s)
    return n((T, D), 1.0), n((F, D), 1.5 / D ** 0.5), n((F, D), 1 / D ** 0.5), n((D, F), 1 / F ** 0.5), n((T, D), 1.0)


@pytest.mark.parametrize("act", gated.ACTS)
@pytest.mark.parametrize("T,D,F", [(3, 264, 200), (40, 72, 136), (100, 128, 264), (300, 200, 392)])
def test_step_within_the_bounds(act, T, D, F):
    X, Wg, Wu, Wd, dY = _normals(T, D, F, T + len(act))
    b = Block(T, D, F, act, X, Wg, Wu, Wd, dY)
    b.fwd()
    b.bwd()
    b.check()
    f = gated.forward(X, Wg, Wu, Wd, act)
    _within(b.Y.t, f.Y, f.err_Y, "Y")
    for k, (v, e) in gated.backward(X, Wg, Wu, Wd, dY, act).items():
        _within(b.out[k].t, v, e, k)


@pytest.mark.parametrize("act", gated.ACTS)
def test_activation_in_its_tails(act):
    """One column of X drives the gate from far below to far above 0: H = act(g), read through Wd = 1."""
    g = np.concatenate([np.linspace(-60, 60, 121), [-1e4, -300.0, -88.0, 0.0, 88.0, 300.0, 1e4]])
    g = gated.rne_bf16(g)
    T = len(g)
    X = np.zeros((T, 8)); X[:, 0] = g; X[:, 1] = 1.0   # noqa: E702
    Wg, Wu, Wd = np.zeros((8, 8)), np.zeros((8, 8)), np.zeros((8, 8))
    Wg[0, 0] = Wu[0, 1] = Wd[0, 0] = 1.0
    for rows in (slice(0, T), slice(0, 40)):            # the kernel for long operands and the one for few tokens
        x = X[rows]
        b = Block(len(x), 8, 8, act, x, Wg, Wu, Wd, training=False)
        b.fwd()
        b.check()
        ref = gated.act(act, x[:, 0])[0]
        # evaluation in float32, one rounding for H (Y = H); results below float32's smallest normal may be flushed
        tol = gated.U16 * np.abs(ref) + gated.ELEM * (1 + np.abs(x[:, 0])) * np.abs(ref) + 2.0 ** -125
        _within(b.Y.t[:, 0], ref, tol, act)
        assert not f32(b.Y.t)[:, 1:].any()


@pytest.mark.parametrize("T", [3, 200])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
def test_gates_whose_square_is_infinite(act, T):
    """Gates of +- 2^66 with U = 1: H, act'(G) and so every gradient are exact: zero, or a power of two times at most T."""
    D, F, big, tiny = 8, 16, 2.0 ** 66, 2.0 ** -20
    X, Wg, Wu, Wd, dY = np.zeros((T, D)), np.zeros((F, D)), np.zeros((F, D)), np.zeros((D, F)), np.zeros((T, D))
    X[:, 0], X[:, 1], Wu[:, 1], dY[:, 2] = big, 1.0, 1.0, tiny
    Wg[:8, 0], Wg[8:, 0], Wd[2, 0], Wd[2, 8] = 1.0, -1.0, 1.0, 1.0
    b = Block(T, D, F, act, X, Wg, Wu, Wd, dY)
    b.fwd()
    b.bwd()
    b.check()
    on = np.zeros(F); on[0] = tiny                         # dH is that for features 0 and 8, whose gates are on and off   # noqa: E702
    Y = np.zeros((T, D)); Y[:, 2] = big   # noqa: E702
    dX = np.zeros((T, D)); dX[:, 0], dX[:, 1] = tiny, tiny * big   # noqa: E702
    _same(b.Y.t, Y, "Y")
    _same(b.out["dX"].t, dX, "dX")
    _same(b.out["dWg"].t, np.outer(on, X.sum(0)), "dWg")
    _same(b.out["dWu"].t, np.outer(on * big, X.sum(0)), "dWu")
    _same(b.out["dWd"].t, np.outer(dY.sum(0), np.repeat([big, 0.0], 8)), "dWd")


def test_buffers_side_by_side():
    """Outputs that touch an input without sharing a byte are taken."""
    T, D, F = 20, 64, 128
    X, Wg, Wu, Wd, dY = _normals(T, D, F, 11)
    apart = Block(T, D, F, "silu", X, Wg, Wu, Wd, dY)
    apart.fwd()
    apart.bwd()
    shapes = [(T, D), (T, D), (F, D), (F, D), (F, D), (F, D), (D, F), (D, F), (T, D), (T, D)]     # X Y Wg dWg Wu dWu Wd dWd dY dX
    room, views = torch.empty(sum(a * c for a, c in shapes), dtype=torch.bfloat16, device="cuda"), []
    for s in shapes:
        views.append(room[:s[0] * s[1]].view(s))
        room = room[s[0] * s[1]:]
    x, y, wg, dwg, wu, dwu, wd, dwd, dy, dx = views
    for v, a in zip((x, wg, wu, wd, dy), (X, Wg, Wu, Wd, dY)):
        v.copy_(_dev(a))
    ctx, ws = binding.alloc_gated_ffn_buffers(apart.desc)
    binding.sf_gated_ffn_fwd(apart.desc, x, wg, wu, wd, y, ctx, ws)
    binding.sf_gated_ffn_bwd(apart.desc, dy, x, wg, wu, wd, ctx, dx, dwg, dwu, dwd, ws)
    assert np.array_equal(bits(y), bits(apart.Y.t))
    for k, v in zip(GRADS, (dx, dwg, dwu, dwd)):
        assert np.array_equal(bits(v), bits(apart.out[k].t)), k
    with pytest.raises(binding.SparseFFNError):
        binding.sf_gated_ffn_bwd(apart.desc, dy, x, wg, wu, wd, ctx, dy, dwg, dwu, dwd, ws)       # the gradient in place


def test_left_out_outputs():
    T, D, F = 70, 72, 136
    b = Block(T, D, F, "silu", *_normals(T, D, F, 5))
    b.fwd()
    b.bwd()
    whole = {k: bits(b.out[k].t) for k in GRADS}
    for only in [("dX",), ("dWg",), ("dWu", "dX"), ("dWd",), ("dWg", "dWd"), ()]:
        for k in GRADS:
            b.out[k].t.fill_(7.0)
        b.bwd(only)
        for k in GRADS:
            if k in only:
                assert np.array_equal(bits(b.out[k].t), whole[k]), (only, k)
            else:
                assert bool((b.out[k].t == 7.0).all()), (only, k)
    b.check()


def test_no_tokens():
    D, F = 64, 72
    z = np.zeros
    b = Block(0, D, F, "silu", z((0, D)), z((F, D)), z((F, D)), z((D, F)), z((0, D)))
    b.fwd()
    for k in GRADS[1:]:
        b.out[k].t.fill_(3.0)
    b.bwd()
    b.check()
    for k in GRADS[1:]:
        assert not bool(b.out[k].t.any())


def test_non_finite_rows_stay_in_their_rows():
    for T in (9, 140):
        D, F = 72, 136
        X, Wg, Wu, Wd, dY = _normals(T, D, F, 9)
        clean = Block(T, D, F, "silu", X, Wg, Wu, Wd, dY)
        clean.fwd()
        X[4, 3], X[6, 5] = np.nan, np.inf
        b = Block(T, D, F, "silu", X, Wg, Wu, Wd, dY)
        b.fwd()
        b.check()
        y, c = f32(b.Y.t), f32(clean.Y.t)
        ok = np.ones(T, bool)
        ok[[4, 6]] = False
        assert np.array_equal(y[ok], c[ok]) and not np.isfinite(y[~ok]).any()


@pytest.mark.parametrize("T", [5, 200])
def test_captured_replayed_and_on_another_stream(T):
    D, F = 136, 264
    a, c = _normals(T, D, F, 11), _normals(T, D, F, 12)
    want = []
    for x in (a, c):
        b = Block(T, D, F, "gelu_tanh", *x)
        b.fwd()
        b.bwd()
        want.append({"Y": bits(b.Y.t), **{k: bits(b.out[k].t) for k in GRADS}})
    s = torch.cuda.Stream()
    b = Block(T, D, F, "gelu_tanh", *a)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        b.fwd()
        b.bwd()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            b.fwd()
            b.bwd()
    s.synchronize()
    for i, x in ((0, a), (1, c), (0, a)):
        for t, v in zip((b.X, b.Wg, b.Wu, b.Wd, b.dY), x):
            t.copy_(_dev(v))
        for g in (b.Y, *b.out.values()):
            g.t.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.check()
        assert np.array_equal(bits(b.Y.t), want[i]["Y"])
        for k in GRADS:
            assert np.array_equal(bits(b.out[k].t), want[i][k]), k
    # the stream handed over instead of made current
    b.Y.t.zero_()
    torch.cuda.synchronize()
    b.fwd(stream=s)
    s.synchronize()
    assert np.array_equal(bits(b.Y.t), want[0]["Y"])


@pytest.mark.parametrize("T", [6, 300])
def test_two_calls_at_once(T):
    """Two streams, each with buffers of its own, forward and backward interleaved."""
    D, F = 264, 520
    data = [_normals(T, D, F, s) for s in (31, 32)]
    want = []
    for x in data:
        b = Block(T, D, F, "silu", *x)
        b.fwd()
        b.bwd()
        want.append([bits(b.Y.t)] + [bits(b.out[k].t) for k in GRADS])
    blocks, streams = [Block(T, D, F, "silu", *x) for x in data], [torch.cuda.Stream() for _ in data]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(blocks, streams):
            b.fwd(stream=s)
        for b, s in zip(blocks, streams):
            b.bwd(stream=s)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        b.check()
        assert all(np.array_equal(x, y) for x, y in zip([bits(b.Y.t)] + [bits(b.out[k].t) for k in GRADS], w))


def test_first_call_inside_a_capture():
    """Nothing has run before in the process: what a first call looks up and sets is allowed while a stream is captured."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import torch
from paper_2602_06183_b200 import binding as b
bf = torch.bfloat16
def block(T):
    D, F = 136, 264
    g = torch.Generator("cuda").manual_seed(T)
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(bf)
    d = b.make_gated_desc(T, D, F)
    t = [n(T, D), n(T, D), n(F, D), n(F, D), n(D, F)]
    out = [torch.zeros_like(x) for x in (t[1], t[1], t[2], t[3], t[4])]
    ctx, ws = b.alloc_gated_ffn_buffers(d)
    def run():
        b.sf_gated_ffn_fwd(d, *t[1:], out[0], ctx, ws)
        b.sf_gated_ffn_bwd(d, *t, ctx, *out[1:], ws)
        q = b.sf_fp4_quantize(t[2][:, :128], b.SF_FP4_NV, 2.0, out=qw)
        x = b.sf_fp4_quantize(t[1][:, :128], b.SF_FP4_NV, 2.0, out=qx)
        b.sf_gemm_fp4(*x, *q, b.SF_FP4_NV, 0.25, C_out=C, workspace=ws4)
    qw = torch.zeros((F, 64), dtype=torch.uint8, device="cuda"), torch.zeros((b.sf_fp4_sizes(F, 128, 0)[1],), dtype=torch.uint8, device="cuda")
    qx = torch.zeros((T, 64), dtype=torch.uint8, device="cuda"), torch.zeros((b.sf_fp4_sizes(T, 128, 0)[1],), dtype=torch.uint8, device="cuda")
    C, ws4 = torch.zeros((T, F), dtype=bf, device="cuda"), torch.zeros((256,), dtype=torch.uint8, device="cuda")
    return run, out + [C]
for T in (5, 200):
    run, out = block(T)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in out]
    for x in out:
        x.zero_()
    run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) and bool(x.any()) for x, y in zip(out, got)), T
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]


def test_repeated_calls_give_the_same_bits():
    for T, D, F in [(1, 4096, 520), (3, 520, 4096), (100, 1024, 1032), (300, 264, 2048)]:
        b = Block(T, D, F, "silu", *_normals(T, D, F, 3))
        got = []
        for _ in range(3):
            b.fwd()
            b.bwd()
            got.append([bits(b.Y.t)] + [bits(b.out[k].t) for k in GRADS])
        b.check()
        for g in got[1:]:
            assert all(np.array_equal(x, y) for x, y in zip(g, got[0]))


@pytest.mark.parametrize("T", [20, 300])
def test_stage_trace(T):
    D, F = 136, 264
    b = Block(T, D, F, "silu", *_normals(T, D, F, 21))
    b.fwd()
    b.bwd()
    want = [bits(b.Y.t)] + [bits(b.out[k].t) for k in GRADS]
    with binding.StageTrace(16) as tr:
        b.fwd()
        b.bwd()
    assert tr.count == 7 and all(ms >= 0 for ms in tr.durations_ms())
    b.check()
    assert all(np.array_equal(x, y) for x, y in zip([bits(b.Y.t)] + [bits(b.out[k].t) for k in GRADS], want))
    with binding.StageTrace(16) as tr:
        b.bwd(("dWg",))
    assert tr.count == 4


def test_offsets_beyond_32_bits():
    """[T, F] of 2.3e9 elements: the last tokens' results are those of a batch of their own (small integers, exact in any order)."""
    T, D, F, tail = 140_000, 64, 16384, 200
    r = np.random.default_rng(4)
    W = [_dev(_ints(s, r, -1, 1)) for s in ((F, D), (F, D))] + [_dev(_ints((D, F), r, -1, 1, 0.05))]
    x, dy = _dev(_ints((tail, D), r)), _dev(_ints((tail, D), r, -1, 1))

    def step(X, dY):
        d = binding.make_gated_desc(len(X), D, F, binding.SF_ACT_RELU)
        ctx, ws = binding.alloc_gated_ffn_buffers(d)
        Y, dX = torch.empty_like(X), torch.empty_like(X)
        g = [torch.empty_like(w) for w in W]
        binding.sf_gated_ffn_fwd(d, X, *W, Y, ctx, ws)
        binding.sf_gated_ffn_bwd(d, dY, X, *W, ctx, dX, *g, ws)
        assert binding.sf_check_status(ws) == binding.SF_OK
        return Y, dX, g
    small = step(x, dy)
    X, dY = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
    X[-tail:], dY[-tail:] = x, dy
    Y, dX, g = step(X, dY)
    assert torch.equal(Y[-tail:], small[0]) and torch.equal(dX[-tail:], small[1])
    assert not bool(Y[:-tail].any()) and not bool(dX[:-tail].any())
    assert all(torch.equal(a, b) for a, b in zip(g, small[2]))          # every other token is zero


@pytest.mark.parametrize("T", [9, 70, 300])
def test_left_out_outputs_in_every_form(T):
    """Sums of two terms, few tokens, CTA pairs: which outputs are asked for changes neither the others' bits nor memory that was not asked for."""
    D, F = 72, 136
    b = Block(T, D, F, "silu", *_normals(T, D, F, 5))
    b.fwd()
    b.bwd()
    whole = {k: bits(b.out[k].t) for k in GRADS}
    for mask in range(15):
        only = tuple(k for i, k in enumerate(GRADS) if mask >> i & 1)
        for k in GRADS:
            b.out[k].t.fill_(7.0)
        b.bwd(only)
        for k in GRADS:
            if k in only:
                assert np.array_equal(bits(b.out[k].t), whole[k]), (only, k)
            else:
                assert bool((b.out[k].t == 7.0).all()), (only, k)
    b.check()
