"""The orthogonalised update through the C ABI, against the iteration in 64 bits.

Bound, in the 2-norm: the final rounding (2^-8 at most) and twice what the operands' roundings do, which the oracle computes by making
them (``orthogonalize_rounded``: float32 sums let a rounding fall the other way, which is as far again at most)."""
import numpy as np
import pytest
import torch

from oracle import around, f32_to_bf16
from paper_2602_06183_b200 import binding as b
from util import Guarded, f32, to_dev

pytestmark = pytest.mark.gpu
BF, U16 = torch.bfloat16, 2.0 ** -8


def _dev(a, dtype=BF):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t if dtype is torch.float32 else to_dev(f32_to_bf16(a.astype(np.float32)).reshape(a.shape))


def _run(G, steps=5, abc=around.ABC, scale=1.0, out=None):
    rows, cols = G.shape
    O, ws = Guarded((rows, cols), BF), Guarded(b.sf_orthogonalize_workspace_size(rows, cols), zero=True)
    o = O.t if out is None else out
    assert b.sf_orthogonalize(G, steps, abc, scale, out=o, workspace=ws.t) is o
    assert b.sf_check_status(ws.t) == b.SF_OK
    O.check("O")
    ws.check("workspace")
    return o


def _check(got, G, steps=5, abc=around.ABC, scale=1.0):
    want = around.orthogonalize(G, steps, abc)
    size = np.linalg.norm(want)
    made = np.linalg.norm(around.orthogonalize_rounded(G, steps, abc) - want)
    off = np.linalg.norm(f32(got).astype(np.float64) / scale - want)
    assert off <= U16 * size + 2 * made, (off / size, made / size)
    assert made < 5e-3 * size                              # the bound is one


def _gradient(m, n, seed=0, rank=None):
    r = np.random.default_rng([m, n, seed])
    if rank:
        return around.rne_bf16(r.normal(size=(m, rank)) @ r.normal(size=(rank, n)))
    return around.rne_bf16(r.normal(size=(m, n)) * 1e-3)


@pytest.mark.parametrize("m,n", [(1, 1), (1, 77), (77, 1), (8, 8), (15, 17), (31, 64), (64, 33), (128, 128), (129, 255), (255, 129), (256, 520), (257, 300),
                                 (300, 257), (520, 1032), (1029, 515), (40, 3001), (3000, 40), (700, 700)])
@pytest.mark.parametrize("dtype", [BF, torch.float32], ids=["bf16", "f32"])
def test_sizes(m, n, dtype):
    G = _gradient(m, n)
    if dtype is torch.float32:
        G = (G * (1 + 1e-4 * np.random.default_rng(m).normal(size=G.shape))).astype(np.float32).astype(np.float64)
    _check(_run(_dev(G, dtype)), G)


@pytest.mark.parametrize("m,n", [(16, 33), (5, 16000), (16, 17000), (33, 4096), (33, 8192), (8200, 33), (64, 100), (90, 96), (96, 2561), (2000, 70), (127, 1030), (128, 1024),
                                 (128, 1025), (4096, 128), (100, 4097), (129, 1024)])
def test_around_the_edges_of_one_launch(m, n):
    """Updates of at most 128 rows (or columns) are made in one launch, in clusters of 1 to 16 CTAs, as long as a warp's columns fit."""
    G = _gradient(m, n, 6)
    _check(_run(_dev(G)), G)


@pytest.mark.parametrize("m,n", [(40, 90), (90, 40), (128, 700), (130, 300)])
def test_steps_one_after_the_other(m, n):
    """k steps and then none differ from k steps by nothing but the result's rounding: every number of them is right."""
    G = _gradient(m, n, 7)
    for steps in range(1, 8):
        _check(_run(_dev(G), steps), G, steps)


@pytest.mark.parametrize("m,n,rank", [(200, 320, 1), (320, 200, 3), (256, 256, 8), (300, 1000, 40)])
def test_low_rank(m, n, rank):
    """Where roundings would grow most: directions of no size are brought up 3.4 times with every step."""
    G = _gradient(m, n, rank=rank)
    _check(_run(_dev(G)), G)


def test_equal_singular_values_and_repeated_rows():
    q = np.linalg.qr(np.random.default_rng(3).normal(size=(96, 96)))[0]
    for G in (around.rne_bf16(np.eye(64, 80) * 3), around.rne_bf16(q), around.rne_bf16(np.tile(q[:1], (40, 1))), np.ones((33, 65))):
        _check(_run(_dev(G)), G)


@pytest.mark.parametrize("steps,abc", [(1, around.ABC), (2, around.ABC), (6, around.ABC), (9, (2.0, -1.5, 0.5)), (7, (1.875, -1.25, 0.375)), (12, (1.5, -0.5, 0.0))])
def test_steps_and_quintics(steps, abc):
    for m, n in ((130, 300), (300, 130)):
        G = _gradient(m, n, 1)
        _check(_run(_dev(G), steps, abc, scale=0.25), G, steps, abc, scale=0.25)


@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -60, 2.0 ** 60, 2.0 ** 120])
def test_size_does_not_matter(size):
    G = _gradient(65, 130, 2) / 2.0 ** -10
    one = _run(_dev(G, torch.float32))
    assert torch.equal(_run(_dev(G * size, torch.float32)), one)
    if size > 2.0 ** -100:
        assert torch.equal(_run(_dev(G * size)), _run(_dev(G)))


def test_zero_nan_and_infinity():
    for shape in ((40, 90), (90, 40)):
        G = torch.zeros(shape, dtype=BF, device="cuda")
        assert not _run(G).any()
        for bad in (float("nan"), float("inf"), -float("inf")):
            G[3, 5] = bad
            assert bool(torch.isnan(_run(G)).all())
    assert b.sf_orthogonalize(torch.zeros((0, 5), dtype=BF, device="cuda")).shape == (0, 5)
    assert b.sf_orthogonalize(torch.zeros((5, 0), dtype=BF, device="cuda")).shape == (5, 0)


@pytest.mark.parametrize("m,n", [(66, 264), (264, 66), (37, 37)])
def test_rows_with_a_stride_and_off_boundaries(m, n):
    G = _gradient(m, n, 4)
    want = _run(_dev(G))
    for pad, off in ((8, 0), (5, 3)):
        for dtype in (BF, torch.float32):
            wide = torch.full((m, n + pad), 9.0, dtype=dtype, device="cuda")
            wide[:, off:off + n] = _dev(G, dtype)
            to = torch.full((m, n + pad), 4.0, dtype=BF, device="cuda")
            assert torch.equal(_run(wide[:, off:off + n], out=to[:, off:off + n]), want) or dtype is torch.float32
            _check(to[:, off:off + n].contiguous(), G)
            rest = torch.ones(n + pad, dtype=torch.bool, device="cuda")
            rest[off:off + n] = False
            assert bool((to[:, rest] == 4).all())


def test_a_transpose_gives_the_transpose():
    G = _dev(_gradient(200, 333, 5))
    assert torch.equal(_run(G), _run(G.T.contiguous()).T)


def test_larger_ones_against_64_bits_on_the_device():
    for m, n in ((1000, 4100), (2300, 1100), (1536, 1536)):
        g = torch.Generator("cuda").manual_seed(m)
        G = (torch.randn(m, 64, generator=g, device="cuda") @ torch.randn(64, n, generator=g, device="cuda") + torch.randn(m, n, generator=g, device="cuda")).to(BF)
        x = G.double() if m <= n else G.double().T
        x = x / x.norm()
        a, bb, c = around.ABC
        for _ in range(5):
            A = x @ x.T
            x = a * x + (bb * A + c * A @ A) @ x
        x = x if m <= n else x.T
        assert float((_run(G).double() - x).norm() / x.norm()) < U16 + 5e-3


def _on_device(G, steps):
    x = G.double() if G.shape[0] <= G.shape[1] else G.double().T
    x = x / x.norm()
    a, bb, c = around.ABC
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (bb * A + c * A @ A) @ x
    return x if G.shape[0] <= G.shape[1] else x.T


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
def test_several_steps_at_once(steps):
    """512 rows and more of a matrix much wider than high: three steps at once, then two at a time. The bound is that of the larger ones above."""
    for m, n in ((1030, 1600), (1700, 1030), (1030, 7300), (13000, 520), (40, 160000), (2100, 5200)):
        g = torch.Generator("cuda").manual_seed(m + steps)
        f = torch.arange(1, 257, device="cuda") ** -0.5
        G = (torch.randn(m, 256, generator=g, device="cuda") * f @ torch.randn(256, n, generator=g, device="cuda") + 0.3 * torch.randn(m, n, generator=g, device="cuda")).to(BF)
        x = _on_device(G, steps)
        for dtype in (BF, torch.float32):
            got = _run(G.to(dtype), steps)
            assert float((got.double() - x).norm() / x.norm()) < U16 + 5e-3
    G = torch.zeros((1024, 7300), dtype=BF, device="cuda")
    assert not _run(G, steps).any()
    G[5, 7] = float("nan")
    assert bool(torch.isnan(_run(G, steps)).all())


@pytest.mark.parametrize("m,n", [(10, 17703), (35, 14517), (9000, 64), (200, 9000), (511, 8000)])
def test_few_rows_of_long_ones_keep_the_precision(m, n):
    """Where several steps at once would lose some: the error is at most 1.5 times that of a result that is rounded only at its end."""
    g = torch.Generator("cuda").manual_seed(m)
    r = min(m, n, 256)
    f = torch.arange(1, r + 1, device="cuda") ** -0.5
    G = ((torch.randn(m, r, generator=g, device="cuda") * f) @ torch.randn(r, n, generator=g, device="cuda") + 0.3 * torch.randn(m, n, generator=g, device="cuda")).to(BF)
    x = _on_device(G, 5)
    once = float((x.to(torch.float32).to(BF).double() - x).norm())
    assert float((_run(G).double() - x).norm()) < 1.5 * once


def test_captured_replayed_on_another_stream_and_side_by_side():
    G = [_dev(_gradient(200, 333, i)) for i in range(2)]
    want = [_run(g) for g in G]
    O = [torch.zeros_like(g) for g in G]
    ws = [torch.zeros(b.sf_orthogonalize_workspace_size(200, 333), dtype=torch.uint8, device="cuda") for _ in G]
    streams = [torch.cuda.Stream() for _ in G]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, s in enumerate(streams):
            b.sf_orthogonalize(G[i], out=O[i], workspace=ws[i], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(O, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.sf_orthogonalize(G[0], out=O[0], workspace=ws[0])
    O[0].zero_()
    g.replay()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(O[0], want[0])
