"""64-bit reference of the operators on 4-bit matrices, from the formats' definitions, in numpy.

Shares no code with the kernels or with the C oracle."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NV, MX = 0, 1


def block_of(fmt):
    return 32 if fmt == MX else 16


def unpack(codes):
    """[rows, cols/2] bytes -> [rows, cols] E2M1 values."""
    c = np.asarray(codes, np.uint8)
    n = np.empty((c.shape[0], 2 * c.shape[1]), np.uint8)
    n[:, 0::2], n[:, 1::2] = c & 15, c >> 4
    return np.where(n & 8, -1.0, 1.0) * GRID[n & 7]


def scale_values(sf, fmt):
    s = np.asarray(sf, np.int64)
    if fmt == MX:
        return np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    e, m = (s >> 3) & 15, s & 7
    v = np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7))
    return np.where((s & 127) == 127, np.nan, v)


def values(codes, sf, fmt, S=1.0):
    """The values a matrix stands for; sf linear [rows, cols/block]."""
    q = unpack(codes)
    return q * np.repeat(scale_values(sf, fmt), block_of(fmt), axis=1) * float(S)


def swizzle(sf):
    """Linear scale codes in the 128x4-atom layout, padding 0."""
    rows, kb = sf.shape
    rb, k4 = -(-rows // 128), -(-kb // 4)
    out = np.zeros(rb * k4 * 512, np.uint8)
    r, k = np.meshgrid(np.arange(rows), np.arange(kb), indexing="ij")
    out[((r // 128) * k4 + k // 4) * 512 + (r % 32) * 16 + (r // 32) % 4 * 4 + k % 4] = sf
    return out


def mxfp4(x):
    """(codes, linear scale codes) of x: X = 2^(floor(log2 m) - 2) per 32, nearest E2M1, ties to the even code."""
    x = np.asarray(x, np.float64)
    y = x.reshape(x.shape[0], -1, 32)
    m = np.abs(y).max(-1)
    fine = np.isfinite(m)
    e = np.where(fine & (m > 0), np.frexp(np.where(fine & (m > 0), m, 1.0))[1] - 1 - 2, -127)
    e = np.maximum(e, -127)
    a = np.abs(np.where(fine[..., None], y, 0.0)) / np.ldexp(1.0, e)[..., None]
    d = np.abs(a[..., None] - GRID)
    near = d.min(-1, keepdims=True)
    tied = d == near
    code = np.where(tied.sum(-1) == 1, tied.argmax(-1),
                    np.where(tied.argmax(-1) % 2 == 0, tied.argmax(-1), tied.argmax(-1) + 1))
    n = (code | np.where(np.signbit(y), 8, 0)).astype(np.uint8).reshape(x.shape)
    return n[:, 0::2] | (n[:, 1::2] << 4), (e + 127).astype(np.uint8)


def random_matrix(rows, cols, fmt, seed, spread=3):
    """Random codes with scales over a few octaves: (codes, linear sf, S or None)."""
    g = np.random.default_rng(seed)
    codes = g.integers(0, 256, (rows, cols // 2)).astype(np.uint8)
    kb = cols // block_of(fmt)
    if fmt == MX:
        return codes, g.integers(127 - spread, 127 + spread + 1, (rows, kb)).astype(np.uint8), None
    return codes, g.integers(56 - 8 * spread, 56 + 8 * spread, (rows, kb)).astype(np.uint8), np.float32(g.uniform(0.01, 0.1))


def act(kind, g):
    """Activation and derivative (0 SiLU, 1 GELU by tanh)."""
    with np.errstate(over="ignore"):
        if kind == 0:
            p = 1 / (1 + np.exp(-g))
            return g * p, p * (1 + g * (1 - p))
        c = np.sqrt(2 / np.pi)
        t = np.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def gated(kind, x, wg, wu):
    g, u = x @ wg.T, x @ wu.T
    return act(kind, g)[0] * u


def gated_grad(kind, x, wg, wu, dh):
    g, u = x @ wg.T, x @ wu.T
    a, da = act(kind, g)
    dg, du = dh * u * da, dh * a
    return dg @ wg + du @ wu, dg.T @ x, du.T @ x
