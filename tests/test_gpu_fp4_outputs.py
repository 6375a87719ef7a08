"""GPU tests of fp4_dequantize into rows of wider buffers, of every type, one row
and several rows a warp."""
import numpy as np
import pytest

from oracle import polyq_fp4_oracle as O
from tests.fp4_util import dense, f64
from tests.test_gpu_fp4_rounding import _once

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [O.MX, O.NV])
@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [5, 20003])
@pytest.mark.parametrize("K,pad,offset", [(300, 0, 0), (300, 3, 1), (304, 8, 8), (301, 4, 4), (1, 2, 1)])
def test_rows_of_wider_buffers(polyq_lib, fmt, t, rows, K, pad, offset):
    """Values of a power of two's tensor scale are exact in fp32 and bf16."""
    rng = np.random.default_rng(K)
    g = 1.0 if fmt == O.MX else 0.25
    codes = rng.integers(0, 16, (rows, K)).astype(np.uint8)
    scales = rng.integers(*((100, 140) if fmt == O.MX else (0, 127)), (rows, -(-K // O.BLOCK[fmt]))).astype(np.uint8)
    q = polyq_lib.Fp4Tensor.pack(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), fmt, g)
    out = dense(rows, K, t, pad, offset)
    polyq_lib.fp4_dequantize(q, out=out)
    v = O.values(codes, scales, fmt, g)
    np.testing.assert_array_equal(f64(out), _once(v, t) if t is torch.float16 else v)
    if pad:
        assert bool(torch.isnan(out.as_strided((rows - 1, pad), (K + pad, 1), offset + K)).all())
    if offset:
        assert bool(torch.isnan(out.as_strided((1, offset), (offset, 1), 0)).all())
