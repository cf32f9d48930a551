"""4-bit operands at the ends of their scales: reading back is bf16(code * sf * alpha) also where code * sf alone leaves float32."""
import numpy as np
import pytest
import torch

from oracle import f32_to_bf16, fp4
from paper_2602_06183_b200 import binding
from util import bits, f32, to_dev

pytestmark = pytest.mark.gpu

FMT = {"nv": binding.SF_FP4_NV, "mx": binding.SF_FP4_MX}


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("alpha", [1.0, 0.25, 2.0 ** -20, 2.0 ** -100, 2.0 ** -149, 2.0 ** 50, 0.3, 1.1e-38, 3.0e38])
def test_read_back_of_every_scale_and_code(fmt, alpha):
    """A row to a scale byte, every code in it. code * sf has three bits, times alpha's 24 it is exact in 64; the path rounds to float32
    once and then to bf16. Results below float32's smallest normal number may be rounded there a second time: half a step of 2^-149."""
    by = np.repeat(np.arange(128 if fmt == "nv" else 256, dtype=np.uint8)[:, None], 64 // fp4.BLOCK[fmt], axis=1)
    codes = np.tile(np.arange(16, dtype=np.uint8), (len(by), 4))
    got = binding.sf_fp4_dequantize(torch.from_numpy(fp4.pack(codes)).cuda(), torch.from_numpy(fp4.tile(by)).cuda(), FMT[fmt], alpha)
    with np.errstate(over="ignore"):
        ref = (fp4.values(codes, by, fmt) * float(np.float32(alpha))).astype(np.float32)
    want = f32_to_bf16(ref).reshape(ref.shape)
    nan = np.isnan(ref)
    g = bits(got)
    assert np.isnan(f32(got)[nan]).all()
    tiny = ~nan & (np.abs(ref) < 2.0 ** -125)
    assert np.array_equal(g[~nan & ~tiny], want[~nan & ~tiny])
    # bf16's subnormal step is 2^-133: half of it, and what float32 lost
    assert np.all(np.abs(f32(got)[tiny].astype(np.float64) - ref[tiny]) <= 2.0 ** -134 + 2.0 ** -149)


@pytest.mark.parametrize("cols", [64, 2048])
@pytest.mark.parametrize("scale", [1.0, 64.0, 2.0 ** 20])
def test_a_block_with_an_infinity_reads_back_as_six_times_its_scale(scale, cols):
    """2^126 is what a block with an infinity gets in the format of powers of two; 6 * 2^126 is beyond float32, 6 * 2^126 / scale is not."""
    x = np.zeros((3, cols), np.float32)
    x[1, 5], x[2, 40] = np.inf, -1e38                      # (the second overflows in its product with the scale, but for scale 1)
    q = binding.sf_fp4_quantize(to_dev(f32_to_bf16(x).reshape(x.shape)), FMT["mx"], scale)
    got = f32(binding.sf_fp4_dequantize(*q, FMT["mx"], 1.0 / scale)).astype(np.float64)
    with np.errstate(over="ignore"):
        codes, by = fp4.quantize(f32_to_bf16(x).reshape(x.shape), "mx", scale)
        want = (fp4.values(codes, by, "mx") / scale).astype(np.float32)
    assert by[1, 0] == 253 and np.array_equal(got, want)
    assert np.isfinite(got).all() or scale == 1.0
