"""Plain 64-bit forms of the layer operators (numpy), for the tests of the kernels."""
import numpy as np

BLOCK = 128


def code_values(codes):
    """The values of e4m3 codes (uint8), without a scale."""
    c = codes.astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, np.ldexp((8 + m).astype(np.float64), e - 10), np.ldexp(m.astype(np.float64), -9))
    v = np.where((c & 0x7f) == 0x7f, np.nan, v)
    return np.where(c >= 128, -v, v)


def nearest_code(x):
    """Nearest e4m3 code of numbers of magnitude 448 or less (ties to even), larger ones to 448."""
    a = np.minimum(np.abs(x), 448.0)
    _, e = np.frexp(np.maximum(a, 2.0 ** -6))
    step = np.ldexp(1.0, e - 4)                   # distance of neighbouring codes in x's binade
    q = np.rint(a / step) * step                  # numpy rounds ties to even
    _, e = np.frexp(np.maximum(q, 2.0 ** -6))
    code = np.where(q >= 2.0 ** -6, ((e + 6) << 3) + np.rint(q / np.ldexp(1.0, e - 4)).astype(np.int64) - 8,
                    np.rint(q * 512).astype(np.int64))
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def block_index(rows, cols, tall):
    return np.arange(rows)[:, None] // tall, np.arange(cols)[None, :] // BLOCK


def pack(x, tall=1):
    """(codes, scale bytes) of a matrix in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nr, nc = -(-rows // tall), -(-cols // BLOCK)
    scales = np.empty((nr, nc), np.uint8)
    codes = np.empty((rows, cols), np.uint8)
    for i in range(nr):
        for j in range(nc):
            b = x[i * tall:(i + 1) * tall, j * BLOCK:(j + 1) * BLOCK]
            at = np.s_[i * tall:(i + 1) * tall, j * BLOCK:(j + 1) * BLOCK]
            if not np.isfinite(b).all():
                scales[i, j] = 255
                codes[at] = 0x7f + 128 * np.signbit(b)
                continue
            most, s = np.abs(b).max(), 7
            while s < 246 and most > 448 * 2.0 ** (s - 127):
                s += 1
            scales[i, j] = s
            codes[at] = nearest_code(b * 2.0 ** (127 - s))
    return codes, scales


def unpack(codes, scales, tall=1):
    i, j = block_index(*codes.shape, tall)
    s = scales[i, j].astype(np.float64)
    return np.where(s == 255, np.nan, code_values(codes) * 2.0 ** (s - 127))


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd):
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, xh
