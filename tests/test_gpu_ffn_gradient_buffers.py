"""GPU tests of the buffers that ffn_backward writes: one weight's gradient as
rows of a wider buffer beside one that the call makes."""
import numpy as np
import pytest

from tests.fp4_util import dense, put

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("given", [0, 1])
@pytest.mark.parametrize("F,pad", [(72, 0), (72, 8), (72, 3), (1, 8)])
def test_one_of_two_is_given(polyq_lib, dtype, given, F, pad):
    """The other gets the given one's type, and is what a call with both gives."""
    rng = np.random.default_rng(F + pad)
    T, K, t = 40, 104, torch.bfloat16
    x, gate, up = (put(rng.standard_normal((r, K)) / 8, t) for r in (T, F, F))
    dh = put(rng.standard_normal((T, F)), t)
    saved = polyq_lib.ffn_saved(T, F)
    polyq_lib.ffn_forward(x, gate, up, saved=saved)
    want = [torch.empty(F, K, dtype=dtype, device="cuda") for _ in range(2)]
    polyq_lib.ffn_backward(x, gate, up, saved, dh, None, *want)
    buffers = [None, None]
    buffers[given] = dense(F, K, dtype, pad)
    got = polyq_lib.ffn_backward(x, gate, up, saved, dh, None, *buffers)
    assert got[1 + given].data_ptr() == buffers[given].data_ptr()
    assert got[1].dtype == got[2].dtype == dtype
    assert torch.equal(got[1], want[0]) and torch.equal(got[2], want[1])
    if pad and F > 1:  # what lies between the rows is not touched
        assert torch.isnan(buffers[given].as_strided((F - 1, pad), (K + pad, 1), K)).all()
