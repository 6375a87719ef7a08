"""The norm's calls in place: an output in the place of an input with another row stride or type
would overwrite rows that are yet to be read, and is refused before anything reaches a GPU."""
import ctypes as C

import pytest

EINVAL = -1
A = 1 << 20  # an aligned address that is never used


def _forward(polyq, x, y, rows=8):
    return polyq._lib.polyq_layernorm_forward(C.byref(x), rows, 128, None, None, 1e-5, 1, C.byref(y), None, None)


def _backward(polyq, x, dy, res, dx, rows=8):
    return polyq._lib.polyq_layernorm_backward(C.byref(x), rows, 128, None, A, 1, C.byref(dy),
                                               None if res is None else C.byref(res), C.byref(dx), None, None, None, 0,
                                               None)


@pytest.mark.parametrize("stride,type_", [(256, 1), (128, 0), (128, 2)])
def test_another_stride_or_type_in_place(polyq_lib, stride, type_):
    base, far = polyq_lib.Dense(A, 128, 1), polyq_lib.Dense(1 << 30, 128, 1)
    other = polyq_lib.Dense(A, stride, type_)
    for a, b in ((base, other), (other, base)):
        assert _forward(polyq_lib, a, b) == EINVAL and "in place" in polyq_lib.last_error()
    assert _backward(polyq_lib, far, other, None, base) == EINVAL and "in place" in polyq_lib.last_error()
    assert _backward(polyq_lib, far, far, other, base) == EINVAL
    if type_ == 1:
        assert "in place" in polyq_lib.last_error()


def test_what_may_lie_in_place_is_not_refused(polyq_lib):
    """One type and stride, or one row; without a GPU the call ends at the device, with one it is not made."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("made-up addresses")
    base, far, wide = (polyq_lib.Dense(a, s, 1) for a, s in ((A, 128), (1 << 30, 128), (A, 256)))
    for rc in (_forward(polyq_lib, base, base), _forward(polyq_lib, base, wide, rows=1),
               _backward(polyq_lib, far, base, None, base), _backward(polyq_lib, far, base, base, base),
               _backward(polyq_lib, far, wide, None, base, rows=1)):
        assert rc not in (0, EINVAL), polyq_lib.last_error()


@pytest.mark.gpu
def test_in_place_equals_out_of_place(polyq_lib):
    import torch
    g = torch.Generator("cuda").manual_seed(1)
    for rows, K in ((300, 512), (7, 1003), (1, 64)):
        x, dy, res = (torch.randn(rows, K, generator=g, device="cuda").bfloat16() for _ in range(3))
        w = torch.randn(K, generator=g, device="cuda")
        stats = polyq_lib.layernorm_stats(rows)
        want = polyq_lib.layernorm_forward(x, w, stats=stats)
        dxs = [polyq_lib.layernorm_backward(x, w, stats, dy, residual=r)[0] for r in (None, res)]
        a, b = dy.clone(), res.clone()
        polyq_lib.layernorm_backward(x, w, stats, a, dx=a)
        polyq_lib.layernorm_backward(x, w, stats, dy, dx=b, residual=b)
        y = x.clone()
        polyq_lib.layernorm_forward(y, w, y=y)
        assert torch.equal(y, want) and torch.equal(a, dxs[0]) and torch.equal(b, dxs[1])
        if rows > 1:
            buf = torch.empty(2 * rows, K, dtype=torch.bfloat16, device="cuda")
            with pytest.raises(polyq_lib.PolyqError):
                polyq_lib.layernorm_forward(buf[:rows], w, y=buf[::2])
