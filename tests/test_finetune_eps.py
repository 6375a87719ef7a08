"""AdamW's eps: subnormal ones, which the kernel's reciprocal takes for 0, are refused."""
import ctypes as C

import pytest

A, EINVAL = 1 << 20, -1


def _step(polyq, eps, lr):
    t = (polyq.AdamwTensor * 1)(polyq.AdamwTensor(A, A, None, 1000, 0, 0.1, 1.0))
    h = polyq.AdamwHyper(lr, 0.9, 0.999, eps, 1, 0, None, None, None)
    s = polyq.AdamwState(A, A, A, A, 1024, 8)
    return polyq._lib.polyq_adamw_step(t, 1, 0, 1, 1, C.byref(s), C.byref(h), None)


@pytest.mark.parametrize("eps", [1e-40, 2.0 ** -127, 2.0 ** -126 * (1 - 2.0 ** -20)])
def test_subnormal_eps(polyq_lib, eps):
    assert _step(polyq_lib, eps, lr=1e-3) == EINVAL


def test_smallest_normal_eps(polyq_lib):
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("made-up addresses")
    assert _step(polyq_lib, 2.0 ** -126, lr=1e-3) not in (0, EINVAL), polyq_lib.last_error()
