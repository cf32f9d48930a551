"""Microscaled 4-bit operands (E2M1 codes with a scale per block). Test infrastructure only.

Formats: "nv" blocks of 16 with E4M3 scales, sf = e4m3(amax / 6); "mx" blocks of 32 with power-of-two scales,
sf = 2^max(floor(log2 amax) - 2, -127). x scale is one float32 product, the two quotients are float32 quotients, a code is the nearest
E2M1 value (ties to the even code, clamped at 6). Scales lie in tiles of 128 rows x 4 blocks.
"""
import numpy as np

from .bf16 import bf16_to_f32
from .fp8 import e4m3_to_f32, f32_to_e4m3

BLOCK = {"nv": 16, "mx": 32}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def f32_to_e2m1(y):
    """Nearest code of a float by search: ties to the even code, clamped, the sign kept (zeros too)."""
    y = np.asarray(y, np.float32)
    a = np.minimum(np.abs(y.astype(np.float64)), 6.0)
    hi = np.clip(np.searchsorted(E2M1, a, side="left"), 0, 7)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - E2M1[lo], E2M1[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return (code | (np.signbit(y).astype(np.int64) << 3)).astype(np.uint8)


def e2m1_to_f64(code):
    v = E2M1[np.asarray(code) & 7]
    return np.where(np.asarray(code) & 8, -v, v)


def scale_value(byte, fmt):
    if fmt == "nv":
        return e4m3_to_f32(byte).astype(np.float64)
    return np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))


def quantize(x_bits, fmt, scale):
    """bf16 patterns [rows, cols] -> (codes [rows, cols], scale bytes [rows, cols / block])."""
    rows, cols = x_bits.shape
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        v = (bf16_to_f32(x_bits) * np.float32(scale)).reshape(rows, -1, BLOCK[fmt])
        nan = np.isnan(v).any(axis=2)
        amax = np.where(nan, np.float32(0), np.abs(np.where(np.isnan(v), np.float32(0), v)).max(axis=2)).astype(np.float32)
        if fmt == "nv":
            by = f32_to_e4m3(amax / np.float32(6))
            by = np.where(nan, np.uint8(0x7F), by)
            sf = e4m3_to_f32(by)
        else:
            e = (amax.view(np.uint32) >> 23).astype(np.int64)
            by = np.where(nan, 255, np.maximum(e - 2, 0)).astype(np.uint8)
            sf = np.ldexp(1.0, by.astype(np.int64) - 127).astype(np.float32)
        s = sf[..., None]
        y = np.where(s > 0, v / np.where(s > 0, s, np.float32(1)), np.copysign(np.float32(0), v))
        y = np.where(np.isnan(y), np.float32(0), y)
    return f32_to_e2m1(y).reshape(rows, cols), by


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def tile_offsets(rows, blocks):
    r, c = np.meshgrid(np.arange(rows), np.arange(blocks), indexing="ij")
    return ((r // 128) * (-(-blocks // 4)) + c // 4) * 512 + 16 * (r % 32) + 4 * (r % 128 // 32) + c % 4


def tile(by, fill=0):
    rows, blocks = by.shape
    out = np.full((-(-rows // 128) * (-(-blocks // 4)) * 512,), fill, np.uint8)
    padded = np.zeros((rows, -(-blocks // 4) * 4), np.uint8)
    padded[:, :blocks] = by
    out[tile_offsets(rows, padded.shape[1])] = padded
    return out


def values(codes, by, fmt):
    rows, cols = codes.shape
    v = e2m1_to_f64(codes).reshape(rows, -1, BLOCK[fmt])
    return (v * scale_value(by, fmt)[..., None]).reshape(rows, cols)
