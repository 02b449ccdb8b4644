"""What stands around a layer, in 64 bits: e4m3 numbers and block scales, norms, gates, residual, the product of e4m3 operands."""
import numpy as np

BLOCK, LEAST, MOST = 128, 2.0 ** -100, 448.0


def e4m3_values():
    """The 256 numbers of the type, by byte (sign, 4 bits of exponent with bias 7, 3 of mantissa; all ones is NaN)."""
    b = np.arange(256)
    e, m = b >> 3 & 15, b & 7
    v = np.where(e > 0, (1 + m / 8) * 2.0 ** (e - 7), m / 8 * 2.0 ** -6)
    v[b & 127 == 127] = np.nan
    return np.where(b & 128, -v, v)


_VALUES = e4m3_values()


def to_e4m3(v):
    """Bytes of the nearest numbers, ties to the even mantissa; beyond 448 is 448, NaN stays."""
    v = np.asarray(v, np.float64)
    grid = _VALUES[:127]
    a = np.minimum(np.abs(v), MOST)
    a = np.where(np.isnan(v), 0.0, a)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    below, above = a - grid[lo], grid[hi] - a
    byte = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    byte = np.where(np.isnan(v), 127, byte) | np.where(np.signbit(v), 128, 0)
    return byte.astype(np.uint8)


def pitch(cols):
    return -(-cols // 512) * 4


def block_amax(x, block_rows):
    """Largest finite magnitude of every block, at least 2^-100."""
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // BLOCK)
    p = np.zeros((nr * block_rows, nc * BLOCK))
    p[:rows, :cols] = np.where(np.isfinite(x), np.abs(x), 0)
    return np.maximum(p.reshape(nr, block_rows, nc, BLOCK).max(axis=(1, 3)), LEAST)


def e8m0_of(amax):
    """Byte of the least power of two s with amax <= 448 s."""
    e = np.ceil(np.log2(amax / MOST) - 1e-12).astype(int)   # then put right where the logarithm is a hair off
    e = np.where(amax > MOST * 2.0 ** e, e + 1, e)
    e = np.where(amax <= MOST * 2.0 ** (e - 1), e - 1, e)
    return e + 127


def spread(s, shape, block_rows):
    return np.repeat(np.repeat(s, block_rows, 0)[:shape[0]], BLOCK, 1)[:, :shape[1]]


def quantize(x, block_rows, e8m0):
    """(bytes, scales as stored: bytes or fp32).  fp32 scales: amax / 448 and 448 / amax are fp32 quotients, and so is the product with x."""
    x = np.asarray(x, np.float64)
    amax = block_amax(x, block_rows)
    if e8m0:
        s = e8m0_of(amax)
        v = x * 2.0 ** (127.0 - spread(s, x.shape, block_rows))
        s = s.astype(np.uint8)
    else:
        a32 = amax.astype(np.float32)
        s = a32 / np.float32(MOST)
        with np.errstate(over="ignore", invalid="ignore"):
            v = (x.astype(np.float32) * spread(np.float32(MOST) / a32, x.shape, block_rows)).astype(np.float64)
    return to_e4m3(np.where(np.isfinite(x), v, np.nan)), s


def scale_values(s):
    return np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127)) if s.dtype == np.uint8 else s.astype(np.float64)


def dequantize(q, s, block_rows):
    return _VALUES[q] * spread(scale_values(s), q.shape, block_rows)


def sigmoid(z):
    return 1 / (1 + np.exp(-z))


def act(z, kind):
    return {"none": lambda: z, "sigmoid": lambda: sigmoid(z), "silu": lambda: z * sigmoid(z)}[kind]()


def norm(x, weight, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight


def residual_norm(x, y, gate, kind, scale, post, pre, eps):
    """(x', h, the part that is added)."""
    u = np.zeros_like(x)
    if y is not None:
        u = y if post is None else norm(y, post, eps)
        if gate is not None:
            u = u * act(gate, kind)
        u = scale * u
    r = x + u
    return r, (r if pre is None else norm(r, pre, eps)), u


def head_norm(o, gate, kind, weight, eps):
    v = o if weight is None else norm(o, weight, eps)
    return v if gate is None else v * act(gate, kind)


def project(xq, xs, wq, ws, widths, bias):
    """Outputs, and the sums of the magnitudes of their products."""
    x, at, block, outs, sizes = dequantize(xq, xs, 1), 0, 0, [], []
    for w in widths:
        n = -(-w // BLOCK)
        W = dequantize(wq[at:at + w], ws[block:block + n], BLOCK)
        outs.append(x @ W.T + (0 if bias is None else bias[at:at + w]))
        sizes.append(np.abs(x) @ np.abs(W).T)
        at, block = at + w, block + n
    return outs, sizes
