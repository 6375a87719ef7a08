"""Pins of the 4-bit floating-point oracle, each against something else: hand
values, brute force over the grid, torch's own e4m3, finite differences."""
import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O

torch = pytest.importorskip("torch")


def test_e4m3_grid_is_torchs():
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(O.E4M3, t)


def test_codes_by_hand():
    """Every border goes to the even code; beyond 6 saturates."""
    v = [0, 0.25, 0.26, 0.5, 0.75, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 5.0, 5.01, 6, 100]
    want = [0, 0, 0.5, 0.5, 1.0, 1.0, 1.5, 2.0, 2.0, 3.0, 4.0, 4.0, 6, 6, 6]
    np.testing.assert_array_equal(O.E2M1[O.nearest_code(np.array(v), O.E2M1)], want)


def test_nearest_by_brute_force():
    rng = np.random.default_rng(1)
    v = np.concatenate([np.abs(rng.standard_normal(2000)) * 3, rng.uniform(0, 460, 2000)])
    for grid in (O.E2M1, O.E4M3):
        np.testing.assert_array_equal(np.abs(v[:, None] - grid).argmin(1), O.nearest_code(v, grid))


def test_mx_block_by_hand():
    x = np.zeros((1, 33))
    x[0, :4] = [7.9, -3.1, 0.3, 1.0]  # floor(log2(7.9)) - 2 = 0: scale 1, 7.9 saturates
    x[0, 32] = 0.1                    # 2^(-4 - 2): 0.1 * 64 = 6.4 -> 6
    codes, scales = O.quantize(x, O.MX)
    np.testing.assert_array_equal(scales, [[127, 121]])
    np.testing.assert_array_equal(O.values(codes, scales, O.MX)[0, [0, 1, 2, 3, 32]],
                                  [6, -3, 0.5, 1, 6 / 64])


def test_nv_block_by_hand():
    x = np.zeros((1, 16))
    x[0, :3] = [12.0, -6.0, 1.1]  # scale 12 / 6 = 2: 6, -3, 0.55 -> 0.5
    codes, scales = O.quantize(x, O.NV)
    np.testing.assert_array_equal(scales, [[(1 + 7) << 3]])
    np.testing.assert_array_equal(O.values(codes, scales, O.NV)[0, :3], [12, -6, 1.0])
    codes, scales = O.quantize(x, O.NV, 2.0)  # the tensor scale moves the block's
    np.testing.assert_array_equal(scales, [[7 << 3]])
    np.testing.assert_array_equal(O.values(codes, scales, O.NV, 2.0)[0, :3], [12, -6, 1.0])


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
def test_quantizing_grid_values_is_exact(fmt):
    rng = np.random.default_rng(3)
    codes = rng.integers(0, 16, (5, 100)).astype(np.uint8)
    codes[codes == 8] = 0
    B = O.BLOCK[fmt]
    codes[:, ::B] = 7  # the block's largest is 6, so its scale comes back
    scales = rng.integers(40, 100, (5, -(-100 // B))).astype(np.uint8)
    v = O.values(codes, scales, fmt)
    c2, s2 = O.quantize(v, fmt)
    np.testing.assert_array_equal(c2, codes)
    np.testing.assert_array_equal(s2, scales)


def test_ffn_gradients_are_differences():
    rng = np.random.default_rng(4)
    p = [rng.standard_normal(s) for s in ((5, 7), (6, 7), (6, 7))]
    dh = rng.standard_normal((5, 6))
    _, a, u = O.ffn(*p)
    for i, g in enumerate(O.ffn_backward(*p, a, u, dh)):
        num = np.zeros_like(p[i])
        for j in np.ndindex(p[i].shape):
            f = []
            for e in (1e-6, -1e-6):
                q = [v.copy() for v in p]
                q[i][j] += e
                f.append((O.ffn(*q)[0] * dh).sum())
            num[j] = (f[0] - f[1]) / 2e-6
        np.testing.assert_allclose(g, num, rtol=1e-6, atol=1e-7)
