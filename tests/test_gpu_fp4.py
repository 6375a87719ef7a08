"""GPU tests of the 4-bit floating-point operators against the fp64 oracle."""
import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O
from tests.fp4_util import check, dense, f64, half_step, put, silu_bound, sum_bound, tiny

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _x(rng, rows, K, kind="plain"):
    x = rng.standard_normal((rows, K)) * np.exp(rng.standard_normal(K))
    if kind == "zeros":  # zero blocks, and a zero row
        x[:, : K // 3] = 0
        x[rows // 2] = 0
    if kind == "tiny":
        x *= 2.0 ** -130
    if kind == "ties":  # exact borders of codes and of scales
        x = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, 6, 4, 0.5], (rows, K)) * \
            rng.choice([-1, 1], (rows, K)) * 2.0 ** rng.integers(-3, 4, (rows, 1))
    return x


def _quantized(polyq, x, fmt, g=1.0, dtype=torch.float32, pad=0):
    t = put(x, dtype, pad)
    return polyq.fp4_quantize(t, fmt, g), f64(t)


def _tensor(polyq, rng, rows, K, fmt):
    """A quantised random tensor and its fp64 values."""
    g = 1.0 if fmt == O.MX else 2.0 ** -6
    q, x = _quantized(polyq, _x(rng, rows, K) * 0.1, fmt, g)
    return q, O.values(*O.quantize(x, fmt, g), fmt, g)


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,K,kind,g,pad", [
    (1, 1, "plain", 1.0, 0), (1, 31, "plain", 1.0, 0), (2, 33, "zeros", 1.0, 3), (3, 256, "ties", 1.0, 0),
    (130, 100, "plain", 0.25, 5), (5, 1027, "plain", 2.0 ** -7, 8), (200, 512, "ties", 2.0, 0),
    (4, 300, "tiny", 1.0, 0), (300, 4096, "zeros", 0.5, 0), (7, 777, "plain", 0.3, 0)])
def test_quantize_matches_oracle(polyq_lib, fmt, dtype, rows, K, kind, g, pad):
    if fmt == O.MX:
        g = 1.0
    if kind == "tiny" and dtype == "f16":
        kind = "plain"
    rng = np.random.default_rng(rows * 1000 + K)
    q, x = _quantized(polyq_lib, _x(rng, rows, K, kind), fmt, g, TYPES[dtype], pad)
    g = float(np.float32(g))
    codes, scales = O.quantize(x, fmt, g)
    gc, gs = (t.cpu().numpy() for t in q.unpack())
    np.testing.assert_array_equal(gs, scales)
    # a negative value that rounds to 0 may keep its sign
    np.testing.assert_array_equal(np.where(gc == 8, 0, gc), codes)
    v = O.values(codes, scales, fmt, g)
    for out in ("f32", "bf16"):
        got = f64(polyq_lib.fp4_dequantize(q, TYPES[out]))
        check(got, v, np.abs(v) * 2 * half_step(TYPES[out]) + tiny(TYPES[out]), out)
        if g in (1.0, 0.25, 0.5, 2.0, 2.0 ** -7) and kind != "tiny":
            np.testing.assert_array_equal(got, v)  # at most 6 significant bits


def test_quantize_odd_last_byte_and_scale_padding(polyq_lib):
    """The upper half of an odd row's last byte and the scales of blocks past a
    row's last are 0, whatever the buffers held."""
    for fmt, K in ((O.MX, 33), (O.NV, 17), (O.NV, 129)):
        t = polyq_lib.Fp4Tensor.empty(3, K, fmt)
        t.codes.fill_(255)
        t.scales.fill_(255)
        polyq_lib.fp4_quantize(torch.ones(3, K, device="cuda"), out=t)
        assert int((t.codes[:, K // 2] >> 4).max()) == 0
        blocks = -(-K // O.BLOCK[fmt])
        pad = t._places(3, -(-blocks // 4) * 4, "cuda")[:, blocks:]
        assert int(t.scales[pad].max()) == 0


def test_quantize_not_finite(polyq_lib):
    """A block with an infinity or a NaN is NaN as a whole, others stay."""
    for fmt in (O.MX, O.NV):
        x = torch.ones(2, 96, device="cuda")
        x[0, 40], x[1, 70] = float("inf"), float("nan")
        v = f64(polyq_lib.fp4_dequantize(polyq_lib.fp4_quantize(x, fmt)))
        B = O.BLOCK[fmt]
        want = O.values(*O.quantize(np.ones((2, 96)), fmt), fmt)
        want[0, 40 // B * B:40 // B * B + B] = np.nan
        want[1, 70 // B * B:70 // B * B + B] = np.nan
        np.testing.assert_array_equal(v, want)


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("rows,K", [(1, 5), (130, 301), (257, 64)])
def test_pack_round_trip(polyq_lib, fmt, rows, K):
    rng = np.random.default_rng(K)
    codes = torch.from_numpy(rng.integers(0, 16, (rows, K)).astype(np.uint8)).cuda()
    scales = torch.from_numpy(rng.integers(100, 126, (rows, -(-K // O.BLOCK[fmt]))).astype(np.uint8)).cuda()
    t = polyq_lib.Fp4Tensor.pack(codes, scales, fmt, 1.0)
    c, s = t.unpack()
    assert torch.equal(c, codes) and torch.equal(s, scales)
    v = O.values(codes.cpu().numpy(), scales.cpu().numpy(), fmt)
    np.testing.assert_array_equal(f64(polyq_lib.fp4_dequantize(t)), v)


SIZES = [  # M, N, K
    (1, 1, 1), (1, 128, 256), (3, 130, 64), (16, 257, 100), (17, 64, 1000), (33, 300, 513), (64, 129, 2050),
    (100, 200, 700), (128, 1000, 300), (129, 100, 64), (256, 256, 256), (256, 300, 260), (300, 131, 333),
    (513, 520, 1100), (130, 2000, 129), (1000, 260, 97)]


def _linear_ref(x, w, res=None):
    y, S = x @ w.T, np.abs(x) @ np.abs(w).T
    return (y, S) if res is None else (y + res, S + np.abs(res))


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_matches_oracle(polyq_lib, fmt, M, N, K):
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    qx, x = _tensor(polyq_lib, rng, M, K, fmt)
    qw, w = _tensor(polyq_lib, rng, N, K, fmt)
    ws = polyq_lib.fp4_workspace()
    y = polyq_lib.fp4_linear(qx, qw, workspace=ws)
    assert polyq_lib.workspace_status(ws) == 0
    ref, S = _linear_ref(x, w)
    check(f64(y), ref, sum_bound(S, K, 64) + 2.0 ** -140, "fp32")


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("M,N,K,pad,offset", [(5, 300, 512, 0, 0), (5, 77, 512, 3, 1), (300, 256, 320, 0, 0),
                                              (300, 200, 320, 8, 8), (300, 77, 320, 3, 1), (513, 600, 64, 1, 0),
                                              (2500, 200, 320, 0, 0), (2500, 136, 320, 4, 4), (2500, 300, 320, 24, 8)])
def test_linear_types_strides_residual(polyq_lib, fmt, dtype, M, N, K, pad, offset):
    rng = np.random.default_rng(M + N + K)
    qx, x = _tensor(polyq_lib, rng, M, K, fmt)
    qw, w = _tensor(polyq_lib, rng, N, K, fmt)
    t = TYPES[dtype]
    res = put(rng.standard_normal((M, N)), t, pad, offset)
    y = dense(M, N, t, pad, offset)
    ref, S = _linear_ref(x, w, f64(res))
    bound = sum_bound(S, K, 64) * 1.01 + np.abs(ref) * half_step(t) + tiny(t)
    polyq_lib.fp4_linear(qx, qw, y=y, residual=res)
    check(f64(y), ref, bound, "residual")
    if pad:  # what lies between the rows is not touched
        assert torch.isnan(y.as_strided((M - 1, pad), (N + pad, 1), offset + N)).all()
    polyq_lib.fp4_linear(qx, qw, y=res, residual=res)  # in place
    assert torch.equal(res, y)


@pytest.mark.parametrize("M", [1, 40, 200])
def test_linear_scale_extremes(polyq_lib, M):
    """Scales from 2^-127 to large ones, zero scales, and a NaN scale that reaches
    its own row only."""
    rng = np.random.default_rng(M)
    K, N = 320, 150
    xc, wc = (rng.integers(0, 16, (r, K)).astype(np.uint8) for r in (M, N))
    xs = rng.integers(0, 256, (M, K // 32)).astype(np.uint8)
    xs[xs == 255] = 0
    ws = (254 - rng.integers(100, 154, (N, K // 32))).astype(np.uint8)
    xs = np.minimum(xs, 150)
    ws[3, 2] = 255
    px = polyq_lib.Fp4Tensor.pack(torch.from_numpy(xc).cuda(), torch.from_numpy(xs).cuda(), O.MX)
    pw = polyq_lib.Fp4Tensor.pack(torch.from_numpy(wc).cuda(), torch.from_numpy(ws).cuda(), O.MX)
    y = f64(polyq_lib.fp4_linear(px, pw))
    x, w = O.values(xc, xs, O.MX), O.values(wc, ws, O.MX)
    assert np.isnan(y[:, 3]).all()
    keep = np.arange(N) != 3
    ref, S = _linear_ref(x, w[keep])
    check(y[:, keep], ref, sum_bound(S, K, 64) + 2.0 ** -126, "extremes")


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("M,F,K", [(1, 1, 1), (1, 128, 256), (2, 130, 700), (16, 300, 100), (30, 257, 513),
                                   (60, 129, 1030), (100, 200, 300), (128, 1000, 64), (129, 128, 64),
                                   (256, 256, 256), (300, 131, 333), (513, 520, 1100), (1000, 260, 97)])
def test_ffn_matches_oracle(polyq_lib, fmt, M, F, K):
    rng = np.random.default_rng(M * 5 + F * 3 + K)
    (qx, x), (qg, g), (qu, u) = (_tensor(polyq_lib, rng, r, K, fmt) for r in (M, F, F))
    h32 = polyq_lib.fp4_ffn(qx, qg, qu, dtype=torch.float32)
    ref, a, b = O.ffn(x, g, u)
    da, du = (sum_bound(np.abs(x) @ np.abs(w).T, K, 64) for w in (g, u))
    bound = silu_bound(a, b, da, du)
    check(f64(h32), ref, bound + 2.0 ** -140, "fp32")
    for t in (torch.bfloat16, torch.float16):
        h = polyq_lib.fp4_ffn(qx, qg, qu, dtype=t)
        check(f64(h), ref, bound * 1.01 + np.abs(ref) * half_step(t) + tiny(t), str(t))
    # the quantised output is fp4_quantize of the fp32 one, bit for bit
    for ofmt, s in ((O.MX, 1.0), (O.NV, 0.125), (O.NV, 0.3)):
        q = polyq_lib.Fp4Tensor.empty(M, F, ofmt, s)
        q.codes.fill_(255)
        q.scales.fill_(255)
        polyq_lib.fp4_ffn(qx, qg, qu, h=q)
        want = polyq_lib.fp4_quantize(h32, ofmt, s)
        for got, exp in zip(q.unpack(), want.unpack()):
            assert torch.equal(got, exp)
        blocks = -(-F // O.BLOCK[ofmt])
        pad = q._places(M, -(-blocks // 4) * 4, "cuda")[:, blocks:]
        assert pad.numel() == 0 or int(q.scales[pad].max()) == 0
        assert F % 2 == 0 or int((q.codes[:, F // 2] >> 4).max()) == 0
