"""Arguments of the 4-bit operators and the gated block that are no tensors are
refused as every other bad argument is, with a ValueError."""
import pytest

torch = pytest.importorskip("torch")

BAD = [7, "buffer", b"bytes", [1], object()]


@pytest.mark.parametrize("bad", BAD, ids=[type(b).__name__ for b in BAD])
def test_no_tensor_for_a_buffer(polyq_lib, bad):
    good = torch.zeros(4, 40, dtype=torch.uint8)
    for call in (lambda: polyq_lib._workspace_at(bad, 0, None, None), lambda: polyq_lib._saved(bad, 4, 8, 0),
                 lambda: polyq_lib.Fp4Tensor(bad, good[0], 4, 8, 0), lambda: polyq_lib.Fp4Tensor(good, bad, 4, 8, 0),
                 lambda: polyq_lib.Fp4Tensor.pack(bad, good), lambda: polyq_lib.Fp4Tensor.pack(good, bad),
                 lambda: polyq_lib.Fp4Tensor.pack(good[0], good)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", BAD, ids=[type(b).__name__ for b in BAD])
def test_no_tensor_for_a_buffer_of_a_call(polyq_lib, bad):
    q = polyq_lib.fp4_quantize(torch.ones(8, 64, device="cuda"))
    h = torch.ones(8, 64, dtype=torch.bfloat16, device="cuda")
    saved = polyq_lib.ffn_saved(8, 8)
    dh = torch.ones(8, 8, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: polyq_lib.fp4_linear(q, q, workspace=bad), lambda: polyq_lib.fp4_linear(q, q, residual=bad),
                 lambda: polyq_lib.fp4_linear(q, q, y=bad), lambda: polyq_lib.fp4_ffn(q, q, q, workspace=bad),
                 lambda: polyq_lib.fp4_ffn(q, q, q, bad), lambda: polyq_lib.fp4_dequantize(q, out=bad),
                 lambda: polyq_lib.fp4_quantize(dh, out=bad), lambda: polyq_lib.ffn_forward(h, h, h, workspace=bad),
                 lambda: polyq_lib.ffn_forward(h, h, h, saved=bad), lambda: polyq_lib.ffn_backward(h, h, h, bad, dh),
                 lambda: polyq_lib.ffn_backward(h, h, h, saved, bad),
                 lambda: polyq_lib.ffn_backward(h, h, h, saved, dh, dgate=bad),
                 lambda: polyq_lib.ffn_backward(h, h, h, saved, dh, workspace=bad)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_a_residual_of_another_type(polyq_lib):
    q = polyq_lib.fp4_quantize(torch.ones(8, 64, device="cuda"))
    res = torch.ones(8, 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        polyq_lib.fp4_linear(q, q, y=torch.empty(8, 8, device="cuda"), residual=res)
    with pytest.raises(ValueError):
        polyq_lib.fp4_linear(q, q, residual=res, dtype=torch.float16)
    assert polyq_lib.fp4_linear(q, q, residual=res).dtype == torch.bfloat16
    assert float(polyq_lib.fp4_linear(q, q, residual=res).max()) == 65
