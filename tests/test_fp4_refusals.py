"""What the entry points of include/polyq_fp4.h refuse before anything reaches a
GPU: every call here has one bad argument beside made-up addresses."""
import ctypes as C
import os
import re

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "polyq_fp4.h")
EINVAL, ENOMEM = -1, -2
A = 1 << 20  # an aligned address that is never used


def _fp4(polyq, **kw):
    d = dict(codes=A, scales=A, rows=64, K=128, code_stride=64, format=0, tensor_scale=1.0)
    d.update(kw)
    return polyq.Fp4Desc(*d.values())


def _dense(polyq, **kw):
    d = dict(data=A, stride=128, type=1)
    d.update(kw)
    return polyq.Dense(*d.values())


def _rc(polyq, name, *args):
    rc = getattr(polyq._lib, name)(*[C.byref(a) if isinstance(a, C.Structure) else a for a in args])
    if rc != 0:
        assert name in polyq.last_error()
    return rc


def test_header_is_bound(polyq_lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(polyq_\w+)\s*\(", text))
    assert len(names) == 10 and names <= set(polyq_lib.exported_symbols())
    zero = int(re.search(r"POLYQ_FP4_WORKSPACE_ZERO (\d+)", text).group(1))
    assert zero == polyq_lib.FP4_WORKSPACE_ZERO


BAD_FP4 = [dict(codes=None), dict(scales=None), dict(codes=A + 8), dict(scales=A + 4), dict(rows=0), dict(K=0),
           dict(rows=-1), dict(rows=(1 << 24) + 1), dict(K=(1 << 24) + 1), dict(code_stride=56),
           dict(code_stride=48), dict(code_stride=0), dict(format=2), dict(format=-1), dict(tensor_scale=0.0),
           dict(tensor_scale=-1.0), dict(tensor_scale=float("inf")), dict(tensor_scale=float("nan")),
           dict(tensor_scale=2.0)]
BAD_DENSE = [dict(data=None), dict(data=A + 1), dict(stride=127), dict(stride=-128), dict(type=3), dict(type=-1)]


@pytest.mark.parametrize("bad", BAD_FP4)
def test_bad_quantised_tensor(polyq_lib, bad):
    t, good = _fp4(polyq_lib, **bad), _fp4(polyq_lib)
    wide = _dense(polyq_lib, stride=1 << 25)
    assert _rc(polyq_lib, "polyq_fp4_quantize", wide, t, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_dequantize", t, wide, None) == EINVAL
    for x, w in ((t, good), (good, t)):
        assert _rc(polyq_lib, "polyq_fp4_linear", x, w, None, wide, A, 1 << 30, None) == EINVAL
    for args in ((t, good, good), (good, t, good), (good, good, t)):
        assert _rc(polyq_lib, "polyq_fp4_ffn", *args, wide, None, A, 1 << 30, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_ffn", good, good, good, None, t, A, 1 << 30, None) == EINVAL


@pytest.mark.parametrize("bad", BAD_DENSE)
def test_bad_dense_tensor(polyq_lib, bad):
    d, q = _dense(polyq_lib, **bad), _fp4(polyq_lib)
    w = _fp4(polyq_lib, rows=128)
    assert _rc(polyq_lib, "polyq_fp4_quantize", d, q, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_dequantize", q, d, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_linear", q, w, None, d, A, 1 << 30, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_linear", q, w, d, _dense(polyq_lib), A, 1 << 30, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_ffn", q, w, w, d, None, A, 1 << 30, None) == EINVAL
    good = _dense(polyq_lib)
    for i in range(4):
        args = [good] * 4
        args[i] = d
        assert _rc(polyq_lib, "polyq_ffn_forward", *args[:3], 64, 128, 128, args[3], None, A, 1 << 30,
                   None) == EINVAL
    for i in range(4):
        args = [good] * 4
        args[i] = d
        assert _rc(polyq_lib, "polyq_ffn_backward", *args[:3], 64, 128, 128, A, args[3], good, None, None,
                   A, 1 << 30, None) == EINVAL
    for grads in ((d, None, None), (None, d, good), (None, good, d)):
        assert _rc(polyq_lib, "polyq_ffn_backward", good, good, good, 64, 128, 128, A, good, *grads,
                   A, 1 << 30, None) == EINVAL


def test_operands_that_do_not_fit(polyq_lib):
    q, y = _fp4(polyq_lib), _dense(polyq_lib, stride=4096)
    for w in (_fp4(polyq_lib, K=96), _fp4(polyq_lib, format=1)):
        assert _rc(polyq_lib, "polyq_fp4_linear", q, w, None, y, A, 1 << 30, None) == EINVAL
        assert _rc(polyq_lib, "polyq_fp4_ffn", q, w, q, y, None, A, 1 << 30, None) == EINVAL
        assert _rc(polyq_lib, "polyq_fp4_ffn", q, q, w, y, None, A, 1 << 30, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_ffn", q, q, _fp4(polyq_lib, rows=65), y, None, A, 1 << 30, None) == EINVAL
    # tensor scales whose product leaves fp32
    for g in (2.0 ** 100, 2.0 ** -100):
        t = _fp4(polyq_lib, format=1, tensor_scale=g)
        assert _rc(polyq_lib, "polyq_fp4_linear", t, t, None, y, A, 1 << 30, None) == EINVAL
        assert _rc(polyq_lib, "polyq_fp4_ffn", t, t, t, y, None, A, 1 << 30, None) == EINVAL
    # one of the two outputs
    out = _fp4(polyq_lib, rows=64, K=64)
    assert _rc(polyq_lib, "polyq_fp4_ffn", q, q, q, None, None, A, 1 << 30, None) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_ffn", q, q, q, y, out, A, 1 << 30, None) == EINVAL
    for bad in (_fp4(polyq_lib, rows=63, K=64), _fp4(polyq_lib, rows=64, K=66)):
        assert _rc(polyq_lib, "polyq_fp4_ffn", q, q, q, None, bad, A, 1 << 30, None) == EINVAL
    # a residual of another type, and y with another stride
    for res in (_dense(polyq_lib, type=0, stride=4096), _dense(polyq_lib, stride=2048)):
        assert _rc(polyq_lib, "polyq_fp4_linear", q, q, res, y, A, 1 << 30, None) == EINVAL


def test_training_block(polyq_lib):
    d, f32 = _dense(polyq_lib), _dense(polyq_lib, type=0)
    f16 = _dense(polyq_lib, type=2)

    def fwd(x=d, g=d, u=d, T=64, F=128, K=128, h=d, saved=A):
        return _rc(polyq_lib, "polyq_ffn_forward", x, g, u, T, F, K, h, saved, A, 1 << 30, None)

    def bwd(x=d, g=d, u=d, T=64, F=128, K=128, saved=A, dh=d, dx=d, dg=d, du=d):
        return _rc(polyq_lib, "polyq_ffn_backward", x, g, u, T, F, K, saved, dh, dx, dg, du, A, 1 << 30, None)

    for call in (fwd, bwd):
        for n in (0, -1, (1 << 24) + 1):
            assert call(T=n) == EINVAL and call(F=n) == EINVAL and call(K=n) == EINVAL
        # 16-bit operands of one type, rows on 16 bytes
        assert call(x=f32, g=f32, u=f32) == EINVAL
        for bad in (f16, f32, _dense(polyq_lib, stride=132), _dense(polyq_lib, data=A + 8)):
            assert call(g=bad) == EINVAL and call(u=bad) == EINVAL
        assert call(x=_dense(polyq_lib, stride=132)) == EINVAL
        assert call(saved=A + 16) == EINVAL
    assert fwd(h=f32) == EINVAL and fwd(h=f16) == EINVAL and bwd(dh=f16) == EINVAL
    assert bwd(saved=None) == EINVAL
    assert bwd(dx=None, dg=None, du=None) == EINVAL
    assert bwd(dg=None) == EINVAL and bwd(du=None) == EINVAL
    assert bwd(dx=f16) == EINVAL and bwd(dg=f16, du=f16) == EINVAL
    assert bwd(dg=f32) == EINVAL and bwd(dg=_dense(polyq_lib, stride=256)) == EINVAL


def test_workspaces(polyq_lib):
    q, d = _fp4(polyq_lib), _dense(polyq_lib)
    for ws, rc in ((None, ENOMEM), (A + 128, EINVAL)):
        assert _rc(polyq_lib, "polyq_fp4_linear", q, q, None, d, ws, 1 << 30, None) == rc
        assert _rc(polyq_lib, "polyq_fp4_ffn", q, q, q, d, None, ws, 1 << 30, None) == rc
        assert _rc(polyq_lib, "polyq_ffn_forward", d, d, d, 64, 128, 128, d, None, ws, 1 << 30, None) == rc
        assert _rc(polyq_lib, "polyq_ffn_backward", d, d, d, 64, 128, 128, A, d, d, None, None, ws, 1 << 30,
                   None) == rc
    n, s = C.c_int64(), C.c_size_t()
    assert _rc(polyq_lib, "polyq_fp4_bytes", 0, 5, 0, C.byref(n), C.byref(n)) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_bytes", 5, 5, 2, C.byref(n), C.byref(n)) == EINVAL
    assert _rc(polyq_lib, "polyq_fp4_bytes", 5, 5, 0, None, C.byref(n)) == EINVAL
    assert _rc(polyq_lib, "polyq_ffn_saved_bytes", 0, 5, C.byref(s)) == EINVAL
    assert _rc(polyq_lib, "polyq_ffn_saved_bytes", 5, 5, None) == EINVAL
    assert _rc(polyq_lib, "polyq_ffn_backward_workspace_bytes", 5, 0, C.byref(s)) == EINVAL


def test_sizes(polyq_lib):
    """Bytes of the layouts, worked by hand."""
    stride, scales = C.c_int64(), C.c_int64()
    for rows, K, fmt, want in ((1, 1, 0, (16, 512)), (128, 33, 0, (32, 512)), (129, 129, 0, (80, 2 * 2 * 512)),
                               (129, 65, 1, (48, 2 * 2 * 512)), (1, 64, 1, (32, 512))):
        assert polyq_lib._lib.polyq_fp4_bytes(rows, K, fmt, C.byref(stride), C.byref(scales)) == 0
        assert (stride.value, scales.value) == want
    n = C.c_size_t()
    assert polyq_lib._lib.polyq_ffn_saved_bytes(3, 33, C.byref(n)) == 0 and n.value == 3 * 64 * 6


def test_scale_layout(polyq_lib):
    """Every (row, block) has a byte of its own inside the buffer, and the
    documented place."""
    torch = pytest.importorskip("torch")
    p = polyq_lib.Fp4Tensor._places(300, 9, "cpu")
    assert p.unique().numel() == 300 * 9 and int(p.max()) < 3 * 3 * 512
    assert int(p[0, 0]) == 0 and int(p[1, 0]) == 16 and int(p[32, 0]) == 4 and int(p[0, 1]) == 1
    assert int(p[0, 4]) == 512 and int(p[128, 0]) == 3 * 512 and int(p[97, 6]) == 512 + 16 + 12 + 2


def test_tensor_scale(polyq_lib):
    """The smallest power of two that keeps amax / 6 / scale within 448."""
    for amax, want in ((2688.0, 1.0), (2689.0, 2.0), (1344.0, 0.5), (1.0, 2.0 ** -11), (0.0, 1.0)):
        assert polyq_lib.fp4_tensor_scale(amax) == want
    for bad in (float("inf"), float("nan"), -1.0):
        with pytest.raises(ValueError):
            polyq_lib.fp4_tensor_scale(bad)


def test_python_refusals(polyq_lib):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    for call in (lambda: polyq_lib.fp4_quantize(x), lambda: polyq_lib.fp4_quantize(None),
                 lambda: polyq_lib.fp4_dequantize(polyq_lib.Fp4Tensor.empty(4, 8, device="cpu")),
                 lambda: polyq_lib.fp4_linear(x, x), lambda: polyq_lib.fp4_ffn(x, x, x),
                 lambda: polyq_lib.ffn_forward(x, x, x),
                 lambda: polyq_lib.Fp4Tensor.pack(torch.zeros(4, 40, dtype=torch.uint8),
                                                  torch.zeros(4, 1, dtype=torch.uint8)),
                 lambda: polyq_lib.Fp4Tensor(torch.zeros(4, 4, dtype=torch.uint8),
                                             torch.zeros(512, dtype=torch.uint8), 4, 8, 0)):
        with pytest.raises(ValueError):
            call()
    for rows, K in ((0, 8), (8, 0)):
        with pytest.raises(polyq_lib.PolyqError):
            polyq_lib.Fp4Tensor.empty(rows, K, device="cpu")


def test_pack_and_unpack_on_the_host(polyq_lib):
    """Codes and scales by hand through the layout (no GPU needed)."""
    torch = pytest.importorskip("torch")
    codes = (torch.arange(3 * 35) % 16).to(torch.uint8).reshape(3, 35)
    scales = torch.tensor([[1, 2], [3, 4], [5, 6]], dtype=torch.uint8)
    t = polyq_lib.Fp4Tensor.pack(codes, scales, polyq_lib.FP4_MX)
    assert t.codes.shape == (3, 32) and int(t.codes[0, 0]) == 0x10 and int(t.codes[0, 17]) == 2
    assert [int(t.scales[i]) for i in (0, 1, 16, 17, 32, 33)] == [1, 2, 3, 4, 5, 6]
    c, s = t.unpack()
    assert torch.equal(c, codes) and torch.equal(s, scales)


@pytest.mark.parametrize("name", ["codes", "scales", "rows", "K", "format", "tensor_scale", "desc", "other"])
def test_fields_are_fixed(polyq_lib, name):
    """A field that changed behind the descriptor would be ignored, or free what it points to."""
    t = polyq_lib.Fp4Tensor.empty(5, 40, polyq_lib.FP4_NV, 0.5, device="cpu")
    with pytest.raises(AttributeError):
        setattr(t, name, getattr(t, name, 1))
    assert (t.rows, t.K, t.format, t.tensor_scale) == (5, 40, polyq_lib.FP4_NV, 0.5)
    again = polyq_lib.Fp4Tensor(t.codes, t.scales, t.rows, t.K, t.format, 0.25)
    assert again.desc.tensor_scale == 0.25 and again.desc.codes == t.desc.codes
