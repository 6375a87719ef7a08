"""GPU tests of the products where the device does not hold every size of thread
block cluster, as a context of few SMs does not: what fits is launched, and
nothing but a call that nothing fits is refused (debug build)."""
import ctypes as C

import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O
from tests.fp4_util import check, f64, half_step, put, silu_bound, sum_bound, tiny

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EUNSUPPORTED, LARGEST = -4, 8


@pytest.fixture
def lib(polyq_lib, polyq_debug):
    """The debug build's entry points behind the binding's functions."""
    for name, (res, args) in polyq_lib._SIGS.items():
        fn = getattr(polyq_debug, name)
        fn.restype, fn.argtypes = res, args
    polyq_debug.polyq_debug_mm_largest_cluster.argtypes = [C.c_int]
    polyq_debug.polyq_debug_mm_largest_cluster.restype = None
    product, polyq_lib._lib = polyq_lib._lib, polyq_debug
    yield polyq_debug.polyq_debug_mm_largest_cluster
    polyq_debug.polyq_debug_mm_largest_cluster(LARGEST)
    polyq_lib._lib = product


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("largest", [1, 2, 3, 7])
def test_products_of_what_fits(polyq_lib, lib, fmt, largest):
    """The split and the kernel change, the sums only in their order."""
    for M, N, K in ((1, 300, 2000), (60, 260, 1500), (300, 257, 700)):
        rng = np.random.default_rng(M)
        (qx, x), (qw, w) = ((polyq_lib.fp4_quantize(put(a, torch.float32), fmt), a) for a in
                            (rng.standard_normal((M, K)), rng.standard_normal((N, K)) / 16))
        x, w = f64(polyq_lib.fp4_dequantize(qx)), f64(polyq_lib.fp4_dequantize(qw))
        lib(largest)
        y, h = polyq_lib.fp4_linear(qx, qw), polyq_lib.fp4_ffn(qx, qw, qw, dtype=torch.float32)
        lib(LARGEST)
        S = np.abs(x) @ np.abs(w).T
        check(f64(y), x @ w.T, sum_bound(S, K, 64) + 2.0 ** -140, "y")
        ref, a, u = O.ffn(x, w, w)
        e = sum_bound(S, K, 64)
        check(f64(h), ref, silu_bound(a, u, e, e) + 2.0 ** -140, "h")


@pytest.mark.parametrize("T", [5, 300])
def test_training_of_what_fits(polyq_lib, lib, T):
    """Single blocks serve the forward pass and dx; the weights' gradients are a
    pair's work and refused by name."""
    rng = np.random.default_rng(T)
    t, F, K = torch.float16, 136, 264
    x, gate, up = (put(rng.standard_normal((r, K)) / 8, t) for r in (T, F, F))
    saved = polyq_lib.ffn_saved(T, F)
    lib(1)
    h = polyq_lib.ffn_forward(x, gate, up, saved=saved)
    dx, _, _ = polyq_lib.ffn_backward(x, gate, up, saved, h, need_weights=False)
    with pytest.raises(polyq_lib.PolyqError, match=r"no cluster .* fits"):
        polyq_lib.ffn_backward(x, gate, up, saved, h)
    lib(LARGEST)
    X, G, U = f64(x), f64(gate), f64(up)
    ref, a, u = O.ffn(X, G, U)
    ea, eu = (sum_bound(np.abs(X) @ np.abs(w).T, K, 16) for w in (G, U))
    check(f64(h), ref, silu_bound(a, u, ea, eu) * 1.01 + np.abs(ref) * half_step(t) + tiny(t), "h")
    again = polyq_lib.ffn_backward(x, gate, up, saved, h)
    # the same da and du, and another order of 2 F products
    da, du = O.act_backward(a, u, f64(h))
    S = np.abs(da) @ np.abs(G) + np.abs(du) @ np.abs(U)
    check(f64(dx), f64(again[0]), 2 * sum_bound(S, 2 * F, 16) * 1.01 + np.abs(f64(dx)) * 2 * half_step(t) + 2 * tiny(t),
          "dx")


def test_nothing_fits(polyq_lib, lib):
    q = polyq_lib.fp4_quantize(torch.ones(4, 64, device="cuda"))
    h = torch.ones(4, 64, dtype=torch.bfloat16, device="cuda")
    ws = polyq_lib.fp4_workspace()
    lib(0)
    for call in (lambda: polyq_lib.fp4_linear(q, q, workspace=ws), lambda: polyq_lib.fp4_ffn(q, q, q, workspace=ws),
                 lambda: polyq_lib.ffn_forward(h, h, h, workspace=ws)):
        with pytest.raises(polyq_lib.PolyqError, match=r"no cluster .* fits") as e:
            call()
        assert e.value.code == EUNSUPPORTED
    lib(LARGEST)
    assert float(polyq_lib.fp4_linear(q, q, workspace=ws).min()) == 64
