"""MXFP4 in 64 bits, from the definition: what the tests of the 4-bit operators compare with."""
import numpy as np
import torch

from paper_1910_06188_b200 import binding as q8

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float32: 2.0 ** -150, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}  # half a step below the normal numbers


def as_numpy(t):
    return t.detach().double().cpu().numpy()


def quantize(x):
    """x [rows, K] (numpy, fp64) -> codes [rows, 32 ceil(K / 32)] as integers, exponents E [rows, ceil(K / 32)]."""
    rows, K = x.shape
    blocks = -(-K // 32)
    v = np.zeros((rows, blocks * 32))
    v[:, :K] = np.where(np.isnan(x), 0.0, x)
    v = v.reshape(rows, blocks, 32)
    top = np.where(np.isinf(v), 0.0, np.abs(v)).max(-1)
    _, e = np.frexp(top)  # top = m 2^e with m in [0.5, 1)
    E = np.where(top == 0, 0, np.maximum(e - 1 - 2 + 127, 0)).astype(np.int64)
    with np.errstate(over="ignore", invalid="ignore"):
        t = np.abs(v) * 2.0 ** (127 - E)[..., None].astype(np.float64)
    below = np.clip(np.searchsorted(GRID, np.minimum(t, 6.0), side="right") - 1, 0, 7)  # the grid point at or below t
    above = np.minimum(below + 1, 7)
    lo, hi = np.minimum(t, 6.0) - GRID[below], GRID[above] - np.minimum(t, 6.0)
    up = (hi < lo) | ((hi == lo) & (above % 2 == 0) & (above != below))  # an even index is an even mantissa
    code = np.where(up, above, below) | (np.signbit(v) * 8)
    return code.reshape(rows, blocks * 32), E


def values(code, E, K):
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (v.reshape(*E.shape, 32) * 2.0 ** (E - 127.0)[..., None]).reshape(code.shape)[:, :K]


def rounded(x):
    """The values that the codes of a tensor's rows stand for, fp64."""
    a = as_numpy(x)
    return values(*quantize(a), a.shape[1])


def unpack(t, group=0):
    """Codes and exponents of a matrix (or one group) from the layout that include/q8.h describes, all columns of its tiles."""
    rows, K = t.shape[-2:]
    row_tiles, k_tiles = -(-rows // 128), -(-K // 256)
    tiles = t.tiles.cpu().numpy()[group * row_tiles * k_tiles * 17408:][:row_tiles * k_tiles * 17408].reshape(row_tiles, k_tiles, 17408)
    b = tiles[:, :, :16384].reshape(row_tiles, k_tiles, 128, 8, 16)
    code = np.empty_like(b)
    for r in range(8):
        for place in range(8):
            code[:, :, r::8, place ^ r] = b[:, :, r::8, place]
    code = np.stack([code & 15, code >> 4], -1).transpose(0, 2, 1, 3, 4, 5).reshape(row_tiles * 128, k_tiles * 256)
    s = tiles[:, :, 16384:].reshape(row_tiles, k_tiles, 2, 32, 4, 4).transpose(0, 4, 3, 1, 2, 5).reshape(row_tiles * 128, k_tiles * 8)
    return code[:rows].astype(np.int64), s[:rows].astype(np.int64), -(-K // 32)


def gelu(y):
    return as_numpy(torch.special.ndtr(torch.from_numpy(y))) * y


def layer(x_hat, w_hat, bias, act, dtype):
    """(y, how far a result may be off it).  A block's 32 products are multiples of 1/4 up to 36 and their sum is exact; the tensor cores then
    add two scaled blocks and the accumulator, 64 columns a time, each addend cut off at no less than 2^-23 of the largest
    partial sum, which sum |x w| bounds: 3 ceil(K / 64) 2^-23 sum |x w|.  The bias is one more fp32 addition; GELU has a slope below
    1.13 and an error of its own below 1e-7 and an fp32 rounding or two; then half a step of the output's type."""
    K = x_hat.shape[1]
    y, total = x_hat @ w_hat.T, np.abs(x_hat) @ np.abs(w_hat).T
    far = 3 * -(-K // 64) * 2.0 ** -23 * total
    if bias is not None:
        b = as_numpy(bias)
        y = y + b
        far = far + 2.0 ** -24 * (np.abs(y) + far)
    if act == q8.Q8_ACT_GELU:
        y, far = gelu(y), 1.13 * far + 1e-7 + 2.0 ** -23 * np.abs(y)
    half = HALF_STEP[dtype]
    return y, far + half * (np.abs(y) + far) + SMALLEST[dtype]


def assert_layer(got, x_hat, w_hat, bias, act):
    y, far = layer(x_hat, w_hat, bias, act, got.dtype)
    off = np.abs(as_numpy(got) - y)
    assert off.shape == y.shape and (off <= far).all(), f"off by {off.max():.3e}, {np.nanmax(off / far):.2f} of what it may be"
