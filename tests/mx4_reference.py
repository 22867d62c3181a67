"""Microscaled 4-bit floating point in 64 bits, from its definition: the reference of the tests."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def quantise(x):
    """fp32-representable rows [rows, K] -> (codes 0..15 [rows, K], scale bytes [rows, K / 32])."""
    x = np.asarray(x, dtype=np.float64)
    rows, K = x.shape
    blocks = x.reshape(rows, K // 32, 32)
    top = np.abs(blocks).max(-1)
    bad = ~np.isfinite(blocks).all(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.where((top > 0) & ~bad, np.frexp(np.where(bad, 1.0, top))[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    v = np.where(bad[..., None], 0.0, np.abs(np.where(np.isfinite(blocks), blocks, 0.0)) / 2.0 ** e[..., None])
    gap = np.abs(v[..., None] - GRID)
    near = gap.min(-1)
    code = np.zeros(v.shape, dtype=np.int64)
    for c in list(range(1, 8, 2)) + list(range(0, 8, 2)):            # an even code last: it wins a tie
        code = np.where(gap[..., c] == near, c, code)
    code = code + 8 * (np.signbit(blocks) & ~bad[..., None])
    byte = np.where(bad, 255, e + 127)
    return code.reshape(rows, K), byte.astype(np.int64)


def values(code, byte):
    v = GRID[code & 7] * np.where(code >= 8, -1.0, 1.0)
    scale = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return v * np.repeat(scale, 32, axis=-1)


def pack_codes(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def pack_scales(byte):
    rows, blocks = byte.shape
    kt = -(-blocks // 4)
    out = np.zeros(-(-rows // 128) * kt * 512, dtype=np.uint8)
    for m in range(rows):
        for b in range(blocks):
            out[((m // 128) * kt + b // 4) * 512 + (m % 32) * 16 + (m // 32 % 4) * 4 + b % 4] = byte[m, b]
    return out.reshape(-(-rows // 128), kt, 512)
