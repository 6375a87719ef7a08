"""GPU tests of what ffn_forward saves for the backward pass: a and u rounded to
nearest, 16 significant bits in fp32's range, in both kernels."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]


def _values(saved, T, F):
    """a and u from the saved planes (upper 16 bits of both, then the next 8)."""
    S = -(-F // 32) * 32
    raw = saved.cpu().numpy()
    hi = raw[:4 * T * S].view(np.uint16).reshape(2, T, S).astype(np.uint32)
    lo = raw[4 * T * S:].reshape(2, T, S).astype(np.uint32)
    return (hi << 16 | lo << 8).view(np.float32)[:, :, :F].astype(np.float64)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,F,K", [(3, 45, 64), (40, 130, 96), (300, 261, 128), (2304, 520, 64)])
def test_to_nearest(polyq_lib, t, T, F, K):
    """Whole numbers below 2^7: every sum is below 2^23, exact in fp32 in any
    order, and saved within half a unit of its 16th bit."""
    rng = np.random.default_rng(T + K)
    x, gate, up = (torch.from_numpy(rng.integers(-127, 128, (r, K)).astype(np.float32)).cuda().to(t)
                   for r in (T, F, F))
    x[0].abs_(), gate[0].abs_()  # sums of 20 bits among them
    saved = polyq_lib.ffn_saved(T, F)
    polyq_lib.ffn_forward(x, gate, up, saved=saved)
    for got, w in zip(_values(saved, T, F), (gate, up)):
        ref = (x.double() @ w.double().T).cpu().numpy()
        half = np.ldexp(1.0, np.frexp(ref)[1] - 17)
        assert (np.abs(got - ref) <= half).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T", [4, 400])
def test_not_finite_and_largest(polyq_lib, t, T):
    """An infinity, a NaN and, of bf16, numbers next to fp32's largest are saved as
    such: a number never becomes an infinity, a NaN never a number."""
    F, K = 40, 64
    x, gate, up = torch.zeros(T, K, dtype=t, device="cuda"), torch.zeros(F, K, dtype=t, device="cuda"), \
        torch.zeros(F, K, dtype=t, device="cuda")
    x[0, 0], x[1, 0], x[2, 0] = float("inf"), float("-inf"), float("nan")
    gate[:, 0], up[:, 0] = 1, 2
    big = t is torch.bfloat16
    if big:  # (2^8 - 1) 2^56 * (2^8 + 2^-..): 0x7F7Fxxxx, its low byte above one half
        x[3, 1:4] = torch.tensor([2.0 ** 64, 2.0 ** 56, 2.0 ** 48], device="cuda")
        gate[:, 1:4] = torch.tensor([255 * 2.0 ** 56, 255 * 2.0 ** 56, 255 * 2.0 ** 56], device="cuda")
    saved = polyq_lib.ffn_saved(T, F)
    polyq_lib.ffn_forward(x, gate, up, saved=saved)
    a, u = _values(saved, T, F)
    for v in (a, u):
        assert (v[0] == np.inf).all() and (v[1] == -np.inf).all() and np.isnan(v[2]).all()
    if big:  # 0x7F7FFFFF in fp32
        top = float(torch.finfo(torch.float32).max)
        assert np.isfinite(a[3]).all() and (np.abs(a[3] - top) <= top * 2.0 ** -15).all()
    assert (a[4:] == 0).all() and (u[4:] == 0).all()
