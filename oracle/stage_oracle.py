"""Plain NumPy forms, in 64 bits and from the definitions, of layer norm with its gradients, of quantization to 8-bit floating
point with a power-of-two scale for each block of 128, and of the product of such operands.  Test infrastructure only."""
import numpy as np

BLOCK = 128
MIN_EXPONENT = -100
E4M3, E5M2 = 0, 1
LARGEST = (448.0, 57344.0)
DIGITS = (3, 2)          # of the fraction
LOWEST = (-6, -14)       # exponent of the smallest normal value


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) of every row."""
    mean = x.mean(axis=1)
    d = x - mean[:, None]
    rstd = 1.0 / np.sqrt((d * d).mean(axis=1) + eps)
    return d * rstd[:, None] * weight + bias, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd):
    """(dx, dweight, dbias)."""
    h = (x - mean[:, None]) * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - h * (g * h).mean(axis=1, keepdims=True))
    return dx, (dy * h).sum(axis=0), dy.sum(axis=0)


def exponent(c, code):
    """The smallest e >= MIN_EXPONENT with c <= LARGEST * 2^e."""
    c = np.asarray(c, dtype=np.float64)
    f, e = np.frexp(np.where(c > 0, c, 1.0) / LARGEST[code])   # c / LARGEST = f * 2^e, 0.5 <= f < 1
    e = np.where(f == 0.5, e - 1, e)
    return np.where(c > 0, np.maximum(e, MIN_EXPONENT), MIN_EXPONENT).astype(np.int64)


def step(v, code):
    """Distance of the code's values around v."""
    _, e = np.frexp(v)
    return np.ldexp(1.0, np.maximum(e - 1, LOWEST[code]) - DIGITS[code])


def nearest(v, code):
    """v (at most LARGEST in magnitude) rounded to the code's nearest value, ties to even."""
    s = step(v, code)
    return np.rint(v / s) * s


def quantize(x, group, code):
    """(values of the codes (rows, cols), exponents (blocks of columns, blocks of `group` rows)) of a finite matrix."""
    rows, cols = x.shape
    up = np.zeros((-(-rows // group) * group, -(-cols // BLOCK) * BLOCK))
    up[:rows, :cols] = x
    tiles = up.reshape(up.shape[0] // group, group, up.shape[1] // BLOCK, BLOCK)
    e = exponent(np.abs(tiles).max(axis=(1, 3)) if tiles.size else np.zeros((tiles.shape[0], tiles.shape[2])), code)
    values = nearest(tiles * np.ldexp(1.0, -e)[:, None, :, None], code).reshape(up.shape)
    return values[:rows, :cols], e.T


def spread(e, rows, cols, group):
    """The scale of every value."""
    return np.ldexp(1.0, e).T.repeat(group, axis=0)[:rows].repeat(BLOCK, axis=1)[:, :cols]


def decode(byte, code):
    """Values of code bytes (E4M3: exponent bias 7, no infinities; E5M2: 15, IEEE style)."""
    byte = np.asarray(byte, dtype=np.int64)
    sign = np.where(byte & 0x80, -1.0, 1.0)
    digits, bias = DIGITS[code], 1 - LOWEST[code]
    field, frac = (byte & 0x7F) >> digits, byte & ((1 << digits) - 1)
    value = np.where(field == 0, np.ldexp(frac.astype(np.float64), LOWEST[code] - digits),
                     np.ldexp(1.0 + frac / float(1 << digits), field - bias))
    if code == E4M3:
        value = np.where((byte & 0x7F) == 0x7F, np.nan, value)
    else:
        value = np.where(field == 31, np.where(frac == 0, np.inf, np.nan), value)
    return sign * value
