"""GPU tests of the roundings that include/polyq_fp4.h promises: the values of a
4-bit tensor are rounded once to the output's type."""
import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O
from tests.fp4_util import dense, f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# significant bits, lowest exponent of a normal number, largest number
FORMS = {torch.bfloat16: (8, -126, (2 - 2.0 ** -7) * 2.0 ** 127), torch.float16: (11, -14, 65504.0)}


def _once(v, t):
    """fp64 values rounded once, to nearest even, to a 16-bit type."""
    bits, low, top = FORMS[t]
    _, e = np.frexp(v)
    q = np.maximum(e - bits, low - bits + 1)
    with np.errstate(over="ignore"):
        r = np.ldexp(np.rint(np.ldexp(v, -q)), q)
        return np.where(np.abs(r) > top, np.copysign(np.inf, v), r)


def _products():
    """Every element code times every finite scale of FP4_NV: exact, at most 6 bits."""
    return np.outer(O.E4M3, np.concatenate([O.E2M1, -O.E2M1]))


def _near_borders(t, n):
    """Tensor scales with which some element lies so near the middle of two
    neighbours of the type that fp32 rounds it there: n normal ones, n among the
    type's smallest numbers."""
    bits, low, _ = FORMS[t]
    rng = np.random.default_rng(bits)
    p = np.unique(_products())
    p = p[p > 0]
    out = []
    while len(out) < 2 * n:
        small = len(out) >= n
        mid = (rng.integers(1, 1 << (bits - 1)) + 0.5) * 2.0 ** (low - bits + 1) if small else \
            (rng.integers(1 << (bits - 1), 1 << bits) + 0.5) * 2.0 ** rng.integers(-9, 3)
        v = p[rng.integers(p.size)]
        g = np.float32(mid / v)
        exact = v * float(g)
        if exact != mid and float(np.float32(v) * g) == mid and _once(exact, t) != _once(mid, t):
            out.append(float(g))
    return out


def _pack(polyq, g, times=1):
    codes = torch.arange(16, dtype=torch.uint8, device="cuda").repeat(127 * times, 1)
    scales = torch.arange(127, dtype=torch.uint8, device="cuda").repeat(times)[:, None]
    return polyq.Fp4Tensor.pack(codes, scales, O.NV, g)


@pytest.mark.parametrize("t", list(FORMS))
def test_values_are_rounded_once(polyq_lib, t):
    """1.5 * 0.1015625 * 0.7676281929016113 is 0.11669921875 in bf16, where fp32
    and then bf16 give 0.1171875; and every element of scales like that one."""
    for g in [0.7676281929016113, 0.3, 1e-45, 2.0 ** -130, 3e38] + _near_borders(t, 20):
        g = float(np.float32(g))
        with np.errstate(over="ignore"):
            want = _once(_products() * g, t)
        q = _pack(polyq_lib, g)
        np.testing.assert_array_equal(f64(polyq_lib.fp4_dequantize(q, t)), want, err_msg=str(g))


@pytest.mark.parametrize("t", list(FORMS))
@pytest.mark.parametrize("times,pad,offset", [(1, 3, 1), (400, 0, 0), (400, 3, 1)])
def test_values_are_rounded_once_in_every_path(polyq_lib, t, times, pad, offset):
    """Rows that start anywhere, several rows a warp."""
    g = _near_borders(t, 1)[0]
    out = dense(127 * times, 16, t, pad, offset)
    polyq_lib.fp4_dequantize(_pack(polyq_lib, g, times), out=out)
    np.testing.assert_array_equal(f64(out), np.tile(_once(_products() * g, t), (times, 1)))


def test_a_nan_scale_stays_nan(polyq_lib):
    for t in FORMS:
        q = polyq_lib.fp4_quantize(torch.full((2, 40), float("nan"), device="cuda"), O.NV, 0.3)
        assert bool(torch.isnan(polyq_lib.fp4_dequantize(q, t)).all())
