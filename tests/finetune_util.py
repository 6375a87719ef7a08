"""Shared by the tests of layer norm, AdamW and the adapters: 64-bit references and
tolerances as arithmetic.  U is half a unit of fp32: what one rounding is off by."""
import numpy as np

from tests.fp4_util import half_step, tiny

U = 2.0 ** -24


def norm(x, w, b, eps, center):
    """y, hat, mean and rstd of fp64 rows."""
    mean = x.mean(1, keepdims=True) if center else np.zeros((len(x), 1))
    c = x - mean
    rstd = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    hat = c * rstd
    return hat * w + b, hat, mean, rstd


def hat_bound(x, hat, rstd, center):
    """Error of hat.  A row's sum adds 8 elements of a thread, then 5 + 5 + 3 levels of a tree (or 8
    blocks in turn): under 26 roundings, with 1/K and its product 28, of the magnitudes; 2 more of
    the difference.  The squares' sum has as many relative ones, twice that of the difference and
    the shift's square; the root halves them; 1/sqrt, eps and the product add four."""
    d = 30 * U * np.abs(x).mean(1, keepdims=True) if center else np.zeros_like(rstd)
    return d * rstd + np.abs(hat) * (24 * U + (d * rstd) ** 2)


def norm_bound(x, w, b, y, hat, rstd, center, dtype):
    return (np.abs(w) * hat_bound(x, hat, rstd, center) + 2 * U * (np.abs(hat * w) + np.abs(b))
            + half_step(dtype) * np.abs(y) * (1 + 2 ** -7) + tiny(dtype))


def norm_backward(x, w, dy, res, eps, center):
    y, hat, mean, rstd = norm(x, w, 0.0, eps, center)
    g = dy * w
    mgh = (g * hat).mean(1, keepdims=True)
    mg = g.mean(1, keepdims=True) if center else np.zeros_like(rstd)
    inner = g - mg - hat * mgh
    return res + rstd * inner, (dy * hat).sum(0), dy.sum(0)


def norm_backward_bounds(x, w, dy, res, eps, center, dtype, vtype):
    """Errors of dx, dw and db: hat's, the sums' (28 roundings over a row; a row each and 20 over
    the rows), four roundings of the inner difference's terms, rstd's 20, the result's."""
    y, hat, mean, rstd = norm(x, w, 0.0, eps, center)
    g, eh = dy * w, hat_bound(x, hat, rstd, center)
    a = np.abs
    mgh, mg = (g * hat).mean(1, keepdims=True), g.mean(1, keepdims=True) * center
    d_mgh = (a(g) * eh).mean(1, keepdims=True) + 31 * U * a(g * hat).mean(1, keepdims=True)
    d_mg = 29 * U * a(g).mean(1, keepdims=True) * center
    terms = a(g) + a(mg) + a(hat * mgh)
    dx = res + rstd * (g - mg - hat * mgh)
    e_dx = (rstd * (d_mg + a(hat) * d_mgh + a(mgh) * eh + 26 * U * terms) + 2 * U * a(res)
            + half_step(dtype) * a(dx) * (1 + 2 ** -7) + tiny(dtype))
    n = len(x) + 20
    e_dw = (a(dy) * eh).sum(0) + n * U * a(dy * hat).sum(0)
    e_db = n * U * a(dy).sum(0)
    dw, db = a((dy * hat).sum(0)), a(dy.sum(0))
    return (e_dx, e_dw + half_step(vtype) * (dw + e_dw) + tiny(vtype),
            e_db + half_step(vtype) * (db + e_db) + tiny(vtype))


# ---- AdamW ----
M32 = np.uint64(0xFFFFFFFF)


def _mix(h):
    h = ((h ^ (h >> np.uint64(16))) * np.uint64(0x9E2D58A5)) & M32
    return ((h ^ (h >> np.uint64(15))) * np.uint64(0x6C62272D)) & M32


def noise(seed, first_block, blocks):
    """The 32 bits of every element of `blocks` blocks of a state, [blocks][256]."""
    b = np.arange(first_block, first_block + blocks, dtype=np.uint64)
    start = _mix(np.array([(seed + 1) & 0xFFFFFFFF], dtype=np.uint64))
    key = _mix(_mix((b & M32) ^ start) ^ (b >> np.uint64(32)) ^ np.uint64(seed >> 32))
    h = _mix((key[:, None] + np.arange(256, dtype=np.uint64) * np.uint64(0x9E3779B1)) & M32)
    return h ^ (h >> np.uint64(16))


def grid(mantissa):
    """The magnitudes of all codes with `mantissa` bits behind 4 exponent bits."""
    one = 1 << mantissa
    c = np.arange(16 * one)
    return np.where(c < one, c / one, (1 + c % one / one) * 2.0 ** (c // one - 1))


def decode(codes, scales, mantissa, signed):
    c = codes.reshape(-1, 256).astype(int)
    v = grid(mantissa)[c & 127 if signed else c] * 2.0 ** (scales.astype(float)[:, None] - 127)
    return np.where(c > 127, -v, v) if signed else v


def scale_of(a, mantissa):
    """Scale byte of blocks of magnitudes: the smallest with which the largest code reaches them."""
    reach = grid(mantissa)[-1] * 2.0 ** (np.arange(255.0) - 127)
    return np.searchsorted(reach, a.max(1), side="left")


def rounded(a, u, mantissa, err, scales):
    """Two values that magnitudes [blocks][256] may be rounded to with 16-bit fractions u when each is
    known up to err: the lower and upper of (a - err, a + err) rounded, in the scales that were
    chosen, which must be those of (a - err) or of (a + err)."""
    assert ((scales == scale_of(np.maximum(a - err, 0), mantissa)) | (scales == scale_of(a + err, mantissa))).all()
    g = grid(mantissa)
    unit = 2.0 ** (scales.astype(float)[:, None] - 127)

    def one(v):
        t = np.maximum(v, 0) / unit
        lo = np.searchsorted(g, t, side="right") - 1
        step = np.diff(g, append=2 * g[-1] - g[-2])
        up = (t - g[lo]) / step[lo] + u / 65536 >= 1
        return g[np.minimum(lo + up, len(g) - 1)] * unit
    return one(a - err), one(a + err), unit * g[1]


def adamw(p, g, m, v, t, lr, b1, b2, eps, decay):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    upd = lr / (1 - b1 ** t) * m / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return p * (1 - lr * decay) - upd, m, v, upd


def adamw_bounds(p, g, m0, v0, upd, pn, m, v, b1, b2, lr, decay, dtype):
    """m: the factors' and products' roundings, of both terms; v: six, all of positive terms; p: that
    of m, half of v's, and of the root, the denominator (2), the quotient (4), the rates (6)."""
    a = np.abs
    e_m = 4 * U * (a(b1 * m0) + a((1 - b1) * g)) + tiny_f32()
    e_v = 6 * U * v + tiny_f32()
    with np.errstate(divide="ignore", invalid="ignore"):
        rel = np.where(m != 0, a(e_m / m), 0) + np.where(v > 0, a(e_v / np.where(v > 0, v, 1)) / 2, 0)
    e_p = a(upd) * (rel + 16 * U) + 4 * U * a(p) + half_step(dtype) * a(pn) * (1 + 2 ** -7) + tiny(dtype)
    return e_p, e_m, e_v


def tiny_f32():
    return 2.0 ** -149


# ---- adapters ----
U32 = 2.0 ** -23


def _split(dtype):
    """What v loses as two 16-bit numbers: relative to itself, and (fp16, scaled by its rows' largest
    magnitude into 2^14 .. 2^15, half a subnormal step of 2^-24) to that magnitude."""
    import torch
    return (2.0 ** -17, 0.0) if dtype == torch.bfloat16 else (2.0 ** -22, 2.0 ** -38)


def adapters(x, a, b, off, ids, scales, ranks, y, dy=None, dx=None, out=None, dxt=None, gt=None):
    """64-bit results of the adapters (torch, any device) and how far a kernel's may be off: lists of
    (value, bound) for y and, with dy, dx, da, db.  y, dx: the residuals (fp64).

    A sum of n products on the tensor cores is off by two units of 2^-23 of the magnitudes for each 16
    of them, and 26 for what adds its parts (8 blocks, 8 warps, ten)."""
    import torch

    def sums(n, s):
        return (2 * (-(-n // 16)) + 26) * U32 * s

    T, K = x.shape
    n, R = a.shape[:2]
    N = b.shape[1]
    rel, floor = _split(x.dtype)
    X, A, B = x.double(), a.double(), b.double()
    Y, EY = y.clone(), torch.zeros_like(y)
    back = dy is not None
    if back:
        D = dy.double()
        DX, EDX = dx.clone(), torch.zeros_like(dx)
        DA, DB = torch.zeros_like(A), torch.zeros_like(B)
        EDA, EDB, LA, LB = (torch.zeros_like(t) for t in (A, B, A, B))
        count = torch.zeros(n, dtype=torch.int64)
    for s0, s1, i in zip(off, off[1:], ids):
        if not 0 <= i < n or s1 <= s0:
            continue
        r, s = int(ranks[i]), float(scales[i])
        t, Ai, Bi = slice(s0, s1), A[i, :r], B[i, :, :r]
        v = X[t] @ Ai.T
        ev = sums(K, X[t].abs() @ Ai.T.abs())
        loss = ev + rel * v.abs() + (floor * v.abs().amax(1, keepdim=True) if r else 0)
        Y[t] += s * v @ Bi.T
        EY[t] += abs(s) * (loss @ Bi.T.abs() + sums(2 * R, v.abs() @ Bi.T.abs()))
        if not back:
            continue
        dv = s * D[t] @ Bi
        edv = abs(s) * sums(N, D[t].abs() @ Bi.abs())
        DX[t] += dv @ Ai
        loss_d = edv + rel * dv.abs()
        EDX[t] += ((loss_d + (floor * dv.abs().amax(1, keepdim=True) if r else 0)) @ Ai.abs()
                   + sums(2 * R, dv.abs() @ Ai.abs()))
        DA[i, :r] += dv.T @ X[t]
        DB[i, :, :r] += s * D[t].T @ v
        if r:
            EDA[i, :r] += (loss_d + floor * dv.abs().max()).T @ X[t].abs()
            EDB[i, :, :r] += abs(s) * D[t].T.abs() @ (ev + rel * v.abs() + floor * v.abs().max())
            LA[i, :r] += dv.T.abs() @ X[t].abs()
            LB[i, :, :r] += abs(s) * D[t].T.abs() @ v.abs()
        count[i] += -(-(s1 - s0) // 64) * 64
    def final(value, e, dtype):
        e = e + 2 * U32 * value.abs()
        return value, e + half_step(dtype) * (value.abs() + e) + tiny(dtype)

    res = [final(Y, EY, out)]
    if back:
        m = int(count.max()) if len(count) else 0
        res += [final(DX, EDX, dxt), final(DA, EDA + sums(2 * m, LA), gt), final(DB, EDB + sums(2 * m, LB), gt)]
    return res
