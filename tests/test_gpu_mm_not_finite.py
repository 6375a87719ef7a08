"""GPU tests of infinities, NaN and extreme block scales in the 4-bit products and
the gated block, in both kernels: what is not finite reaches the outputs that the
formula gives it and no others."""
import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O
from tests.fp4_util import check, f64, sum_bound

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOKENS = [3, 100, 2304]  # few, several tiles of few, pairs


def _pack(polyq, codes, scales, fmt, g=1.0):
    return polyq.Fp4Tensor.pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), fmt, g)


@pytest.mark.parametrize("g", [2.0 ** -120, 3e-37])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quotients_beyond_fp32(polyq_lib, g, dtype):
    """A finite x whose quotient by the tensor scale is infinite makes its block NaN."""
    x = torch.full((3, 64), 2.0 ** -115, device="cuda").to(dtype)
    x[1, 20] = 2.0 ** 20
    q = polyq_lib.fp4_quantize(x, O.NV, g)
    codes, scales = O.quantize(f64(x), O.NV, float(np.float32(g)))
    got = [t.cpu().numpy() for t in q.unpack()]
    assert scales[1, 1] == 0x7F and (np.delete(scales.ravel(), 5) < 0x7F).all()
    np.testing.assert_array_equal(got[0], codes)
    np.testing.assert_array_equal(got[1], scales)
    assert bool(torch.isnan(polyq_lib.fp4_dequantize(q)[1, 16:32]).all())


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("M", TOKENS)
def test_extreme_scales(polyq_lib, fmt, M):
    """Zero scales, the smallest and the largest, and NaN ones: of a weight's row
    they reach a column of y, of a token's a row."""
    rng = np.random.default_rng(M + fmt)
    K, N = 320, 520
    B = O.BLOCK[fmt]
    xc, wc = (rng.integers(0, 16, (r, K)).astype(np.uint8) for r in (M, N))
    if fmt == O.MX:  # pairs of scales from 2^-127 2^-27 to 2^23 2^27
        xs = np.minimum(rng.integers(0, 255, (M, K // B)), 150).astype(np.uint8)
        ws = rng.integers(100, 155, (N, K // B)).astype(np.uint8)
        nan = 255
    else:
        xs, ws = (rng.choice([0, 1, 7, 8, 56, 120, 126], (r, K // B)).astype(np.uint8) for r in (M, N))
        nan = 127
    xs[M // 2, 4], ws[3, 2], ws[N - 1, K // B - 1] = nan, nan, nan
    y = f64(polyq_lib.fp4_linear(_pack(polyq_lib, xc, xs, fmt), _pack(polyq_lib, wc, ws, fmt)))
    x, w = O.values(xc, xs, fmt), O.values(wc, ws, fmt)
    rows, cols = np.arange(M) != M // 2, ~np.isin(np.arange(N), (3, N - 1))
    assert np.isnan(y[~rows]).all() and np.isnan(y[:, ~cols]).all()
    x, w = x[rows], w[cols]
    check(y[rows][:, cols], x @ w.T, sum_bound(np.abs(x) @ np.abs(w).T, K, 64) + 2.0 ** -126, "y")


@pytest.mark.parametrize("M", TOKENS)
def test_gated_block_in_4_bits(polyq_lib, M):
    """Sums beyond fp32 and NaN scales in x, gate and up: the dense output is the
    formula's, the quantised one is fp4_quantize of it."""
    F, K = 264, 64
    xc, gc, uc = (np.full((r, K), 2, np.uint8) for r in (M, F, F))  # ones
    xs, gs, us = (np.full((r, K // 32), 121, np.uint8) for r in (M, F, F))  # 2^-6
    xs[0] = 254  # sums of 64 2^127 2^-6, one half of which is fp32's largest power of two
    xs[1, 0] = 255
    gc[5], gc[70], uc[6], uc[71] = 10, 0, 10, 0  # minus ones and zeros
    gs[200, 1], us[201, 0] = 255, 255
    gs[9], us[10] = 127, 127  # these leave fp32 with token 0
    x, g, u = (_pack(polyq_lib, c, s, O.MX) for c, s in ((xc, xs), (gc, gs), (uc, us)))
    h = polyq_lib.fp4_ffn(x, g, u, dtype=torch.float32)
    with np.errstate(all="ignore"):
        v = [O.values(c, s, O.MX) for c, s in ((xc, xs), (gc, gs), (uc, us))]
        a, b = ((v[0] @ w.T).astype(np.float32) for w in v[1:])
        ref = (a / (1 + np.exp(-a)).astype(np.float32)) * b
        got = h.cpu().numpy()
        np.testing.assert_array_equal(np.isnan(got), np.isnan(ref))
        inf = np.isinf(ref)
        assert inf.any() and np.isnan(ref).any()
        np.testing.assert_array_equal(got[inf], ref[inf])
        rest = np.isfinite(ref)
        assert np.allclose(got[rest], ref[rest], rtol=(8 + 1.2 * 64) * 2.0 ** -23, atol=0)
    for fmt, s in ((O.MX, 1.0), (O.NV, 2.0 ** 100)):
        q = polyq_lib.Fp4Tensor.empty(M, F, fmt, s)
        polyq_lib.fp4_ffn(x, g, u, h=q)
        for p, r in zip(q.unpack(), polyq_lib.fp4_quantize(h, fmt, s).unpack()):
            assert torch.equal(p, r)


def _train(polyq, x, gate, up, dh):
    T, F = x.shape[0], gate.shape[0]
    saved = polyq.ffn_saved(T, F)
    h = polyq.ffn_forward(x, gate, up, saved=saved)
    return (h, *polyq.ffn_backward(x, gate, up, saved, dh))


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", TOKENS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_training_block(polyq_lib, t, T, value):
    F, K, at, f = 200, 136, T - 1, 131
    g = torch.Generator("cuda").manual_seed(T)
    x, gate, up = ((torch.randn(r, K, generator=g, device="cuda") / 8).to(t) for r in (T, F, F))
    dh = torch.randn(T, F, generator=g, device="cuda").to(t)
    base = _train(polyq_lib, x, gate, up, dh)
    assert all(bool(torch.isfinite(b).all()) for b in base)
    tokens, feats = torch.arange(T, device="cuda") != at, torch.arange(F, device="cuda") != f
    # in one gradient of h: its token's dx, its feature's gradients
    d = dh.clone()
    d[at, f] = value
    h, dx, dgate, dup = _train(polyq_lib, x, gate, up, d)
    assert torch.equal(h, base[0])
    assert torch.equal(dx[tokens], base[1][tokens]) and not bool(torch.isfinite(dx[at]).any())
    for got, ref in ((dgate, base[2]), (dup, base[3])):
        assert torch.equal(got[feats], ref[feats]) and not bool(torch.isfinite(got[f]).any())
    # in a token: its h and dx; every gradient of the weights
    d = x.clone()
    d[at, 7] = value
    h, dx, dgate, dup = _train(polyq_lib, d, gate, up, dh)
    assert torch.equal(h[tokens], base[0][tokens]) and torch.equal(dx[tokens], base[1][tokens])
    a, u = (d[at].double() @ w.double().T for w in (gate, up))
    ref = (a / (1 + torch.exp(-a)) * u).to(t)
    assert torch.equal(torch.isnan(h[at]), torch.isnan(ref)) and not bool(torch.isfinite(h[at]).any())
    assert torch.equal(h[at].nan_to_num(0, 1, -1), ref.nan_to_num(0, 1, -1))
    assert not bool(torch.isfinite(dgate[:, 7]).any()) and not bool(torch.isfinite(dup[:, 7]).any())
    # in a row of gate: its feature's h, and all of dx
    w = gate.clone()
    w[f, 7] = value
    h, dx, dgate, dup = _train(polyq_lib, x, w, up, dh)
    assert torch.equal(h[:, feats], base[0][:, feats]) and torch.equal(dup[feats], base[3][feats])
    a = x.double() @ w[f].double()
    ref = (a / (1 + torch.exp(-a)) * (x.double() @ up[f].double())).to(t)
    assert torch.equal(h[:, f].nan_to_num(0, 1, -1), ref.nan_to_num(0, 1, -1))
    assert torch.equal(dgate[feats], base[2][feats]) and not bool(torch.isfinite(dx[:, 7]).any())


@pytest.mark.parametrize("M", TOKENS)
def test_far_negative_gates(polyq_lib, M):
    """silu within (8 + 1.2 |a|) 2^-23 of its value down to a = -87, and between
    that value and 0 below, where exp(-a) leaves fp32."""
    F, K = 96, 96  # a = -(f + 1): ones in the first f + 1 columns of gate
    t = torch.bfloat16
    x = torch.ones(M, K, device="cuda", dtype=t)
    gate = -torch.tril(torch.ones(F, K, device="cuda", dtype=t))
    up = torch.zeros(F, K, device="cuda", dtype=t)
    up[:, 0] = 1
    q = [polyq_lib.fp4_quantize(v, O.MX) for v in (x, gate, up)]
    h = f64(polyq_lib.fp4_ffn(*q, dtype=torch.float32))
    a = -np.arange(1.0, F + 1)
    ref = a / (1 + np.exp(-a))
    near = a >= -87
    assert (np.abs(h - ref)[:, near] <= (np.abs(ref) * (8 + 1.2 * np.abs(a)) * 2.0 ** -23)[near]).all()
    far = ref[~near] * (1 + 2.0 ** -15)
    assert far.size and ((h[:, ~near] >= far) & (h[:, ~near] <= 0)).all()
