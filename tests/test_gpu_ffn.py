"""GPU tests of the 16-bit gated feed-forward block and its gradients."""
import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O
from tests.fp4_util import U32, check, dense, f64, half_step, put, silu_bound, sum_bound, tiny

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16]


def _inputs(rng, T, F, K, t, pad=0):
    x = put(rng.standard_normal((T, K)), t, pad + (-K) % 8)
    gate, up = (put(rng.standard_normal((F, K)) / np.sqrt(K), t, pad + (-K) % 8) for _ in range(2))
    return x, gate, up


def _values(saved, T, F):
    """a and u as fp64 from the saved planes (upper 16 bits of both, then the next 8)."""
    S = -(-F // 32) * 32
    raw = saved.cpu().numpy()
    hi = raw[:4 * T * S].view(np.uint16).reshape(2, T, S).astype(np.uint32)
    lo = raw[4 * T * S:].reshape(2, T, S).astype(np.uint32)
    return (hi << 16 | lo << 8).view(np.float32)[:, :, :F].astype(np.float64)


def _forward_ref(x, gate, up, K):
    h, a, u = O.ffn(x, gate, up)
    da, du = (sum_bound(np.abs(x) @ np.abs(w).T, K, 16) for w in (gate, up))
    return h, a, u, da, du


SIZES = [  # T, F, K
    (1, 1, 1), (1, 128, 64), (5, 130, 72), (17, 200, 1000), (64, 257, 100), (128, 128, 128), (129, 64, 8),
    (256, 256, 192), (300, 131, 330), (515, 264, 520), (130, 1000, 40)]


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,F,K", SIZES)
def test_forward(polyq_lib, t, T, F, K):
    rng = np.random.default_rng(T * 3 + F * 5 + K)
    x, gate, up = _inputs(rng, T, F, K, t)
    saved = polyq_lib.ffn_saved(T, F, t)
    ws = polyq_lib.fp4_workspace()
    h = polyq_lib.ffn_forward(x, gate, up, saved=saved, workspace=ws)
    assert polyq_lib.workspace_status(ws) == 0
    ref, a, u, da, du = _forward_ref(f64(x), f64(gate), f64(up), K)
    check(f64(h), ref, silu_bound(a, u, da, du) * 1.01 + np.abs(ref) * half_step(t) + tiny(t), "h")
    for n, got, ref, e in zip("au", _values(saved, T, F), (a, u), (da, du)):
        check(got, ref, e * 1.01 + np.abs(ref) * 2.0 ** -15 + 2.0 ** -140, n)
    assert torch.equal(h, polyq_lib.ffn_forward(x, gate, up))


def _backward_bounds(x, gate, up, a, u, dh, t, K):
    """References from the saved a, u, and bounds: da and du are computed to
    (12 + 1.2 |a|) units and rounded to half a step, sums are fp32."""
    da, du = O.act_backward(a, u, dh)
    s = 1 / (1 + np.exp(-a))
    mag = np.abs(dh * u) * s * (1 + np.abs(a))  # 1 + a (1 - s) may cancel
    ea = mag * (12 + 1.2 * np.abs(a)) * U32 * 1.01 + np.abs(da) * half_step(t) * 1.001 + tiny(t)
    eu = np.abs(du) * ((12 + 1.2 * np.abs(a)) * U32 + half_step(t)) * 1.01 + tiny(t)
    T, F = a.shape
    dx = da @ gate + du @ up
    ex = ea @ np.abs(gate) + eu @ np.abs(up) + \
        sum_bound(np.abs(da) @ np.abs(gate) + np.abs(du) @ np.abs(up), 2 * F, 16) * 1.01
    eg = ea.T @ np.abs(x) + sum_bound(np.abs(da).T @ np.abs(x), T, 16) * 1.01
    ep = eu.T @ np.abs(x) + sum_bound(np.abs(du).T @ np.abs(x), T, 16) * 1.01
    return (dx, ex), (da.T @ x, eg), (du.T @ x, ep)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("T,F,K", SIZES)
def test_backward(polyq_lib, t, T, F, K):
    rng = np.random.default_rng(T * 3 + F * 7 + K)
    x, gate, up = _inputs(rng, T, F, K, t)
    dh = put(rng.standard_normal((T, F)), t)
    saved = polyq_lib.ffn_saved(T, F, t)
    polyq_lib.ffn_forward(x, gate, up, saved=saved)
    a, u = _values(saved, T, F)
    refs = _backward_bounds(f64(x), f64(gate), f64(up), a, u, f64(dh), t, K)
    ws = polyq_lib.ffn_workspace(T, F)
    got = polyq_lib.ffn_backward(x, gate, up, saved, dh, workspace=ws)
    assert polyq_lib.workspace_status(ws) == 0
    for n, g, (ref, e) in zip(("dx", "dgate", "dup"), got, refs):
        check(f64(g), ref, e * 1.01 + np.abs(ref) * half_step(t) + tiny(t), n)
    # fp32 gradients, rows of wider buffers
    outs = [dense(r, K, torch.float32, 5) for r in (T, F, F)]
    polyq_lib.ffn_backward(x, gate, up, saved, dh, *outs)
    for n, g, (ref, e) in zip(("dx", "dgate", "dup"), outs, refs):
        check(f64(g), ref, e + 2.0 ** -140, n + " fp32")
    only = polyq_lib.ffn_backward(x, gate, up, saved, dh, need_weights=False)
    assert only[1] is None and only[2] is None and torch.equal(only[0], got[0])
    only = polyq_lib.ffn_backward(x, gate, up, saved, dh, need_dx=False)
    assert only[0] is None and torch.equal(only[1], got[1]) and torch.equal(only[2], got[2])


@pytest.mark.parametrize("t", TYPES)
def test_strides_and_views(polyq_lib, t):
    """x, gate and up as rows of wider buffers; gate and up halves of one
    matrix; h and dh with odd strides."""
    rng = np.random.default_rng(5)
    T, F, K = 200, 136, 264
    w = put(rng.standard_normal((2 * F, K)) / 16, t, 16)
    x = put(rng.standard_normal((T, K)), t, 24, 8)
    gate, up = w[:F], w[F:]
    dh = put(rng.standard_normal((T, F)), t, 3, 1)
    h = dense(T, F, t, 5, 1)
    saved = polyq_lib.ffn_saved(T, F, t)
    polyq_lib.ffn_forward(x, gate, up, h=h, saved=saved)
    saved2 = polyq_lib.ffn_saved(T, F, t)
    c = [v.contiguous() for v in (x, gate, up, dh)]
    assert torch.equal(h, polyq_lib.ffn_forward(c[0], c[1], c[2], saved=saved2))
    got = polyq_lib.ffn_backward(x, gate, up, saved, dh)
    for p, q in zip(got, polyq_lib.ffn_backward(c[0], c[1], c[2], saved2, c[3])):
        assert torch.equal(p, q)


def test_gradients_against_differences(polyq_lib):
    """Along random directions, the gradients agree with differences of the
    block in 64 bits.  The operators' values differ from the fp64 gradient by
    16-bit roundings of a, u, da, du and the results: each of the sums below is
    a dot product with a random direction, so six relative half steps of the sum
    of magnitudes bound it; the central difference's own error is of order e^2."""
    rng = np.random.default_rng(11)
    t, T, F, K = torch.float16, 150, 140, 96
    x, gate, up = _inputs(rng, T, F, K, t)
    dh = put(rng.standard_normal((T, F)), t)
    saved = polyq_lib.ffn_saved(T, F, t)
    polyq_lib.ffn_forward(x, gate, up, saved=saved)
    grads = polyq_lib.ffn_backward(x, gate, up, saved, dh)
    base, d64 = [f64(v) for v in (x, gate, up)], f64(dh)
    e = 1e-5
    _, a, u = O.ffn(*base)
    for i, g in enumerate(grads):
        v = rng.standard_normal(base[i].shape)
        f = []
        for s in (e, -e):
            p = list(base)
            p[i] = p[i] + s * v
            f.append(float((O.ffn(*p)[0] * d64).sum()))
        diff = (f[0] - f[1]) / (2 * e)
        got = float((f64(g) * v).sum())
        da, du = O.act_backward(a, u, d64)
        if i == 0:
            mag = np.abs(da) @ np.abs(base[1]) + np.abs(du) @ np.abs(base[2])
        else:
            mag = np.abs(da if i == 1 else du).T @ np.abs(base[0])
        assert abs(got - diff) <= 6 * half_step(t) * float((mag * np.abs(v)).sum()) + 1e-6 * abs(diff)


def test_saved_beyond_fp16(polyq_lib):
    """Values beyond fp16's range are saved as they are.  Their gradients may
    leave it too: dup = sum over 4 tokens of (2^-10 * 320000) * 100 = 125000, so
    they are taken in fp32."""
    T, F, K = 4, 16, 64
    x = torch.full((T, K), 100.0, dtype=torch.float16, device="cuda")
    gate = torch.full((F, K), 50.0, dtype=torch.float16, device="cuda")
    up = torch.zeros(F, K, dtype=torch.float16, device="cuda")
    saved = polyq_lib.ffn_saved(T, F, torch.float16)
    h = polyq_lib.ffn_forward(x, gate, up, saved=saved)
    a, u = _values(saved, T, F)
    assert (a == 320000).all() and (u == 0).all() and (h == 0).all()
    dx, dgate, dup = (torch.empty(r, K, device="cuda") for r in (T, F, F))
    polyq_lib.ffn_backward(x, gate, up, saved, torch.full_like(h, 2.0 ** -10), dx, dgate, dup)
    assert (dx == 0).all() and (dgate == 0).all() and (dup == 125000).all()
