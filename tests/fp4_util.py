"""Shared by the tests of the 4-bit operators and the gated block: dense rows of
any stride, 64-bit references and the tolerances, as arithmetic.

A product's sum is in fp32 on the tensor cores: every instruction adds 64 (4-bit)
or 16 (16-bit) exact products and the running sum, taken as two roundings of at
most one unit in the last place (2^-23) of the sum of magnitudes S; the cluster's
parts (up to 8), the residual and the scale add ten more.  A result's rounding is
half a unit of its type."""
import numpy as np

U32 = 2.0 ** -23


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def tiny(dtype):
    """Half the spacing of a type's subnormals."""
    import torch
    f = torch.finfo(dtype)
    return f.tiny * f.eps / 2


def dense(rows, cols, dtype, pad=0, offset=0, fill=float("nan"), device="cuda"):
    """A [rows][cols] tensor whose rows are `pad` elements wider and start
    `offset` elements into their buffer; the rest holds `fill`."""
    import torch
    buf = torch.full((rows * (cols + pad) + offset,), fill, dtype=dtype, device=device)
    return buf[offset:].view(rows, cols + pad)[:, :cols]


def put(a, dtype, pad=0, offset=0):
    """A NumPy matrix on the GPU in such a tensor."""
    import torch
    t = dense(*a.shape, dtype, pad, offset)
    t.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return t


def f64(t):
    return t.detach().double().cpu().numpy()


def sum_bound(S, K, per):
    """Error of an fp32 sum of K products with sum of magnitudes S."""
    return (2 * (-(-K // per)) + 10) * U32 * S


def check(got, ref, bound, what=""):
    got = np.asarray(got, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.isfinite(got).all(), f"{what}: not finite"
    bad = np.abs(got - ref) > bound
    if bad.any():
        i = np.unravel_index(np.argmax(np.abs(got - ref) - bound), got.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} off, worst at {i}: "
                             f"{got[i]!r} against {ref[i]!r}, bound {bound[i]!r}")


def silu_bound(a, u, da, du):
    """Error of silu(a) * u from errors da, du of its factors and of expf's fast
    form (2 + 1.16 |a| units), the quotient and the product (6 more); |silu'| < 1.1."""
    h = np.abs(a / (1 + np.exp(-a)) * u)
    return 1.1 * da * (np.abs(u) + du) + np.abs(a) * du + h * (8 + 1.2 * np.abs(a)) * U32
