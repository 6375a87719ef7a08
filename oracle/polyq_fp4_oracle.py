"""Plain fp64 restatement of the 4-bit floating-point formats and of the gated
feed-forward block (NumPy only, shares no code with the library).

An e2m1 code is sign, two exponent bits and one mantissa bit; MX blocks are 32
elements with a power-of-two scale, NV blocks 16 elements with an e4m3 scale
and a scale per tensor.
"""
import numpy as np

MX, NV = 0, 1
BLOCK = {MX: 32, NV: 16}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3_values():
    """The 127 finite non-negative e4m3 numbers, in code order."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(out)


E4M3 = e4m3_values()


def nearest_code(v, grid):
    """Index of the grid value nearest to each v >= 0; of two equally near ones
    the even index; the last one beyond the grid."""
    v = np.asarray(v, np.float64)
    hi = np.clip(np.searchsorted(grid, v), 1, len(grid) - 1)
    lo = hi - 1
    dl, dh = v - grid[lo], grid[hi] - v
    return np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)


def quantize(x, fmt, g=1.0):
    """(codes uint8 [rows][K], scale bytes uint8 [rows][blocks]) of fp32-exact x."""
    x = np.asarray(x, np.float64)
    rows, K = x.shape
    B = BLOCK[fmt]
    n = -(-K // B)
    t = np.zeros((rows, n * B))
    with np.errstate(over="ignore", invalid="ignore"):
        t[:, :K] = x if fmt == MX else (x / g).astype(np.float32)
    t = t.reshape(rows, n, B)
    a = np.abs(t)
    bad = ~np.isfinite(t).all(2)
    a = np.where(bad[:, :, None], 0.0, a)
    top = a.max(2)
    if fmt == MX:
        _, e = np.frexp(top)  # top = m 2^e, m in [1/2, 1)
        byte = np.where(top > 0, np.clip(e - 1 - 2, -127, 127) + 127, 0)
        s = 2.0 ** (byte - 127.0)
        byte = np.where(bad, 255, byte)
    else:
        byte = nearest_code((top / 6).astype(np.float32), E4M3)
        s = E4M3[byte]
        byte = np.where(bad, 0x7F, byte)
    q = nearest_code(a / np.where(s > 0, s, np.inf)[:, :, None], E2M1)
    q = q + 8 * (np.signbit(t) & (q > 0))
    return q.reshape(rows, -1)[:, :K].astype(np.uint8), byte.astype(np.uint8)


def values(codes, scales, fmt, g=1.0):
    """fp64 values of codes and scale bytes."""
    codes = np.asarray(codes)
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    sb = np.asarray(scales).astype(np.int64)
    if fmt == MX:
        s = np.where(sb == 255, np.nan, 2.0 ** (sb - 127.0))
    else:
        s = np.where(sb == 0x7F, np.nan, E4M3[np.minimum(sb, 126)])
    return v * np.repeat(s, BLOCK[fmt], axis=1)[:, :codes.shape[1]] * g


def silu(a):
    return a / (1 + np.exp(-a))


def ffn(x, gate, up):
    """(h, a, u) of the gated block."""
    a, u = x @ gate.T, x @ up.T
    return silu(a) * u, a, u


def act_backward(a, u, dh):
    """(da, du)."""
    s = 1 / (1 + np.exp(-a))
    return dh * u * s * (1 + a * (1 - s)), dh * a * s


def ffn_backward(x, gate, up, a, u, dh):
    """(dx, dgate, dup)."""
    da, du = act_backward(a, u, dh)
    return da @ gate + du @ up, da.T @ x, du.T @ x
