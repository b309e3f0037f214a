"""The 4-bit microscaled format from its definition, in numpy and 64 bits, for the tests of the layer
operators: encoding, stored layout, decoding."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def encode(x):
    """x (rows x cols, any float type) -> (codes rows x 32 nb, scale bytes rows x nb)."""
    x = np.asarray(x).astype(np.float64)
    rows, cols = x.shape
    nb = -(-cols // 32)
    v = np.zeros((rows, nb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, nb, 32)
    finite = np.isfinite(v).all(2)
    top = np.where(finite[:, :, None], np.abs(v), 0).max(2)
    exp = np.where(top > 0, np.frexp(np.where(top > 0, top, 1))[1] - 1 - 2, -127)
    exp = np.maximum(exp, -127)
    with np.errstate(invalid="ignore"):
        u = np.where(finite[:, :, None], np.abs(v), 0) / np.exp2(exp.astype(np.float64))[:, :, None]
    # nearest of the eight magnitudes, a tie to the even code
    mags = VALUES[:8]
    code = np.zeros(u.shape, np.uint8)
    for c in range(1, 8):
        mid = (mags[c - 1] + mags[c]) / 2
        code = np.where((u > mid) | ((u == mid) & (c % 2 == 0)), c, code).astype(np.uint8)
    code |= (np.signbit(v).astype(np.uint8) << 3)
    code[~finite] = 0
    scale = np.where(finite, exp + 127, 255).astype(np.uint8)
    return code.reshape(rows, nb * 32), scale


def scale_offsets(rows, cols):
    """Byte of the scale of every (row, block)."""
    nb = -(-cols // 32)
    r, j = np.arange(rows)[:, None], np.arange(nb)[None, :]
    return ((r // 128) * (-(-cols // 256)) + j // 8) * 1024 + j % 8 // 4 * 512 + r % 32 * 16 + r % 128 // 32 * 4 + j % 4


def pack(codes, scales, cols, fill=0):
    """Stored bytes; `fill` goes where the layout leaves the scale bytes open (rows behind the last)."""
    rows = codes.shape[0]
    packed = (codes[:, 0::2] | (codes[:, 1::2] << 4)).reshape(-1)
    out = np.full(-(-rows // 128) * -(-cols // 256) * 1024, fill, np.uint8)
    out[scale_offsets(rows, -(-cols // 256) * 256)] = 0
    out[scale_offsets(rows, cols)] = scales
    return packed, out


def decode(codes, scales, cols):
    """FP64 values, rows x cols."""
    rows, nb = scales.shape
    v = VALUES[codes].reshape(rows, nb, 32) * np.exp2(scales.astype(np.float64) - 127)[:, :, None]
    v = np.where((scales == 255)[:, :, None], np.nan, v)
    return v.reshape(rows, nb * 32)[:, :cols]


def quantised(x):
    """x's values after the round trip."""
    return decode(*encode(x), np.asarray(x).shape[1])
