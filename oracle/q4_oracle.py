"""Oracle of the 4-bit matrices, in numpy, from the definitions: MX4 blocks of 32 with a power-of-two scale, NV4 blocks of
16 with an e4m3 scale and a power of two for the whole matrix, codes e2m1, nearest, ties to the even code.  All in 64 bits but one step: NV4's
scale comes from a product in fp32 with the fp32 number 1 / (6 g), as the format defines it (`exact_scale_byte` has the quotient of real arithmetic,
to judge that step by).  Shares nothing with the library but the layout of a quantised matrix, which include/dc.h fixes."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 3) for e in range(-6, 9) for m in range(8)][:-1])
MX4, NV4 = 0, 1


def block_of(fmt):
    return 32 if fmt == MX4 else 16


def nearest(v, grid):
    """Index of the grid point nearest to each v >= 0, ties to the even index, the last one beyond the grid."""
    mid = (grid[1:] + grid[:-1]) / 2              # exact: grid points have few bits
    if len(mid) < 10:                             # few borders: counted one by one, which is faster on large arrays
        n = np.zeros(v.shape, dtype=np.int64)
        for i, m in enumerate(mid):
            n += v > m if i % 2 == 0 else v >= m  # a border between an even index and the odd one above it belongs to the even one
        return n
    below, upto = np.searchsorted(mid, v, side="left"), np.searchsorted(mid, v, side="right")
    return np.where((below != upto) & (upto % 2 == 0), upto, below)


def quantize(x, fmt, g=1.0):
    """(codes 0..15 [rows, cols], scale bytes [rows, blocks]) of a float array."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    b = block_of(fmt)
    blocks = -(-cols // b)
    pad = np.zeros((rows, blocks * b))
    pad[:, :cols] = x
    v = pad.reshape(rows, blocks, b)
    odd = ~np.isfinite(v).all(-1)
    top = np.where(odd, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(-1))
    if fmt == MX4:
        e = np.frexp(top)[1] - 1 - 2              # floor(log2 top) - 2
        e = np.where(top > 0, np.maximum(e, -127), -127)
        byte, scale = (e + 127).astype(np.int64), np.ldexp(1.0, e)
        byte = np.where(odd, 255, byte)
    else:
        with np.errstate(over="ignore"):
            byte = nearest((np.float32(top) * (np.float32(1) / np.float32(6.0 * g))).astype(np.float64), E4M3)     # in fp32, as the format is defined
        scale = E4M3[byte] * g
        byte = np.where(odd, 127, byte)
    with np.errstate(divide="ignore", invalid="ignore"):
        u = np.where(scale[..., None] > 0, np.abs(v) / scale[..., None], 0.0)
    u = np.where(np.isfinite(u), u, 0.0)
    code = nearest(u, E2M1) + np.where(np.signbit(v), 8, 0)
    code = np.where(odd[..., None], -1, code)     # any code: the block reads as NaN
    return code.reshape(rows, blocks * b)[:, :cols], byte


def exact_scale_byte(top, g):
    """NV4: e4m3 nearest to the quotient top / (6 g) of real arithmetic, 448 at most.  In 64 bits that is on the quotient's side of each border, or on the
    border with it: top has at most 24 bits, and a border times 6 g at most 7."""
    return nearest(np.asarray(top, dtype=np.float64) / (6.0 * g), E4M3)


def scales(byte, fmt, g=1.0):
    if fmt == MX4:
        return np.where(byte == 255, np.nan, np.ldexp(1.0, byte - 127))
    return np.append(E4M3, np.nan)[byte] * g


def values(code, byte, fmt, g=1.0):
    """What codes and scale bytes stand for."""
    rows, cols = code.shape
    s = np.repeat(scales(byte, fmt, g), block_of(fmt), axis=1)[:, :cols]
    return np.where(code > 7, -1.0, 1.0) * E2M1[code & 7] * s


def stands_for(x, fmt, g=1.0):
    return values(*quantize(x, fmt, g), fmt, g)


def unpack(buf, rows, cols, fmt):
    """(codes of all columns a row has room for, scale bytes of all rows and blocks its tiles have room for) of a quantised matrix."""
    b = block_of(fmt)
    pitch = -(-cols // 64) * 32
    tiles = -(-cols // (4 * b))
    off = -(-rows * pitch // 256) * 256
    raw = np.asarray(buf, dtype=np.uint8)
    assert raw.size == off + -(-rows // 128) * tiles * 512
    by = raw[:rows * pitch].reshape(rows, pitch)
    code = np.empty((rows, 2 * pitch), dtype=np.int64)
    code[:, 0::2], code[:, 1::2] = by & 15, by >> 4
    t = raw[off:].reshape(-1, tiles, 32, 4, 4)                         # row tile, tile, row % 32, row % 128 / 32, block % 4
    return code, t.transpose(0, 3, 2, 1, 4).reshape(-1, tiles * 4).astype(np.int64)


def product(xv, wv, bias=None, residual=None, relu6=False, matmul=lambda a, b: a @ b.T):
    """act(X W^T + bias + residual) of values, in 64 bits (`matmul`: a faster a b^T in 64 bits)."""
    y = matmul(xv, wv)
    if bias is not None:
        y = y + np.asarray(bias, dtype=np.float64)
    if residual is not None:
        y = y + np.asarray(residual, dtype=np.float64)
    return np.clip(y, 0.0, 6.0) if relu6 else y
