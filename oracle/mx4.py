"""Packed mx4 matrices on the CPU: the values of a block in the documented fp32 order and in 64 bits, the layout of the bytes, and
products in 64 bits.  Written from the format's description (include/tahq_mx4.h), with none of the library's code."""
import numpy as np

FLOOR, COVER = 0, 1
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
ROOT = np.float32(1 / np.sqrt(32.0))


def blocks(x):
    """[rows, cols] -> [rows, blocks, 32], filled up with zeros."""
    rows, cols = x.shape
    y = np.zeros((rows, -(-cols // 32) * 32), x.dtype)
    y[:, :cols] = x
    return y.reshape(rows, -1, 32)


def rotate(y):
    """(1 / sqrt 32) H_32 on the last axis: butterflies in the order the format names, in y's own type."""
    y = y.copy()
    with np.errstate(all="ignore"):
        for h in (1, 2, 4, 8, 16):
            v = y.reshape(y.shape[:-1] + (16 // h, 2, h))
            a, b = v[..., 0, :].copy(), v[..., 1, :].copy()
            v[..., 0, :], v[..., 1, :] = a + b, a - b
        return y * (ROOT if y.dtype == np.float32 else 1 / np.sqrt(32.0))


def encode(x, transform=0, rule=FLOOR):
    """fp32 [rows, cols] -> (codes uint8 [rows, blocks, 32], scales uint8 [rows, blocks])."""
    y = blocks(np.asarray(x, np.float32))
    if transform:
        y = rotate(y)
    with np.errstate(all="ignore"):
        top = np.abs(y).max(-1)
        bad = ~np.isfinite(y).all(-1)
        mantissa, exponent = np.frexp(np.where(bad, 1.0, top).astype(np.float64))    # top = mantissa 2^exponent, in [1/2, 1)
        e = exponent - 3 + ((mantissa > 0.75) if rule == COVER else 0)
        e = np.where(top > 0, np.maximum(e, -127), -127)
        a = np.abs(np.where(bad[..., None], 0.0, y).astype(np.float64)) / np.exp2(e.astype(np.float64))[..., None]
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    a = np.minimum(np.rint(a / step) * step, 6.0)
    codes = np.searchsorted(GRID, a).astype(np.uint8) | (np.signbit(y).astype(np.uint8) << 3)
    codes[bad] = 0
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def values(codes, scales):
    """The numbers that codes and scales stand for, in 64 bits: [rows, 32 * blocks]."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    with np.errstate(all="ignore"):
        return (v * scale[..., None]).reshape(codes.shape[0], -1)


def packed_size(rows, cols):
    return -(-rows // 32) * (-(-cols // 64) * 1024 + -(-cols // 256) * 256)


def pack(codes, scales, cols):
    """The bytes of the packed matrix, block by block."""
    rows, nb = scales.shape
    RB, KB, KC = -(-rows // 32), -(-cols // 64), -(-cols // 256)
    c = np.zeros((RB * 32, KB * 2, 32), np.uint8)
    c[:rows, :nb] = codes
    pairs = c[..., 0::2] | (c[..., 1::2] << 4)                                        # [row, block, 16 bytes]
    pairs = pairs.reshape(RB, 32, KB, 2, 16).transpose(0, 2, 3, 1, 4)
    s = np.zeros((RB * 32, KC * 8), np.uint8)
    s[:rows, :nb] = scales
    words = s.reshape(RB, 32, KC, 4, 2).transpose(0, 2, 4, 1, 3)                      # [RB, KC, half, row, four units]
    return np.concatenate([pairs.reshape(-1), words.reshape(-1)])


def quantize(x, transform=0, rule=FLOOR):
    """fp32 [rows, cols] -> the packed matrix's bytes."""
    return pack(*encode(x, transform, rule), x.shape[1])


def unpack(packed, rows, cols):
    """Packed bytes -> (codes [rows, blocks, 32], scales [rows, blocks]) of the blocks that hold columns."""
    RB, KB, KC, nb = -(-rows // 32), -(-cols // 64), -(-cols // 256), -(-cols // 32)
    n = RB * KB * 1024
    pairs = packed[:n].reshape(RB, KB, 2, 32, 16).transpose(0, 3, 1, 2, 4).reshape(RB * 32, KB * 2, 16)
    codes = np.empty((RB * 32, KB * 2, 32), np.uint8)
    codes[..., 0::2], codes[..., 1::2] = pairs & 15, pairs >> 4
    words = packed[n:n + RB * KC * 256].reshape(RB, KC, 2, 32, 4).transpose(0, 3, 1, 4, 2).reshape(RB * 32, KC * 8)
    return codes[:rows, :nb], words[:rows, :nb]


def dequantize(packed, rows, cols, transform=0):
    """Packed bytes -> fp32 values, the rotation undone in the documented order."""
    v = values(*unpack(packed, rows, cols)).astype(np.float32)
    if transform:
        v = rotate(v.reshape(rows, -1, 32)).reshape(rows, -1)
    return v[:, :cols]


def matmul(a, b, m, n, k):
    """(A B^T, |A| |B|^T) of two packed matrices in 64 bits; the second is what rounding errors go by."""
    va, vb = values(*unpack(a, m, k)), values(*unpack(b, n, k))
    with np.errstate(all="ignore"):
        return va @ vb.T, np.abs(va) @ np.abs(vb).T
