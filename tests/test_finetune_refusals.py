"""What the entry points of include/polyq_finetune.h refuse before anything reaches a
GPU: every call here has one bad argument beside made-up addresses."""
import ctypes as C
import os
import re

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "polyq_finetune.h")
EINVAL, ENOMEM, EUNSUPPORTED = -1, -2, -4
A = 1 << 20  # an aligned address that is never used
NAN, INF = float("nan"), float("inf")


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
    assert len(names) == 8 and names <= set(polyq_lib.exported_symbols())
    for name in ("ADAMW_BLOCK", "ADAPTERS_WORKSPACE_ZERO"):
        assert int(re.search(rf"POLYQ_{name} (\d+)", text).group(1)) == getattr(polyq_lib, name)


# ---- layer norm ----
def _fwd(polyq, x=None, rows=8, K=128, w=None, b=None, eps=1e-5, y=None, stats=None):
    d = _dense(polyq)
    return _rc(polyq, "polyq_layernorm_forward", x or d, rows, K, w, b, eps, 1, y or d, stats, None)


def _bwd(polyq, x=None, rows=8, K=128, w=None, stats=A, dy=None, res=None, dx="x", dw=None, db=None, ws=A, n=1 << 40):
    d = _dense(polyq)
    return _rc(polyq, "polyq_layernorm_backward", x or d, rows, K, w, stats, 1, dy or d, res,
               d if dx == "x" else dx, dw, db, ws, n, None)


BAD = [dict(data=None), dict(data=A + 1), dict(stride=127), dict(stride=-128), dict(type=3), dict(type=-1)]


@pytest.mark.parametrize("bad", BAD)
def test_norm_of_a_bad_tensor(polyq_lib, bad):
    d, good = _dense(polyq_lib, **bad), _dense(polyq_lib)
    assert _fwd(polyq_lib, x=d) == EINVAL and _fwd(polyq_lib, y=d) == EINVAL
    assert _bwd(polyq_lib, x=d) == EINVAL and _bwd(polyq_lib, dy=d) == EINVAL and _bwd(polyq_lib, dx=d) == EINVAL
    assert _bwd(polyq_lib, res=d) == EINVAL
    if "stride" not in bad:
        assert _fwd(polyq_lib, w=d) == EINVAL and _fwd(polyq_lib, b=d) == EINVAL
        for k in ("w", "dw", "db"):
            assert _bwd(polyq_lib, **{k: d}) == EINVAL
    assert _rc(polyq_lib, "polyq_layernorm_forward", None, 8, 128, None, None, 1e-5, 1, good, None, None) == EINVAL


@pytest.mark.parametrize("n", [0, -1, (1 << 24) + 1])
def test_norm_sizes(polyq_lib, n):
    assert _fwd(polyq_lib, rows=n) == EINVAL and _fwd(polyq_lib, K=n) == EINVAL
    assert _bwd(polyq_lib, rows=n) == EINVAL and _bwd(polyq_lib, K=n) == EINVAL
    size = C.c_size_t()
    for rows, K in ((n, 8), (8, n)):
        assert _rc(polyq_lib, "polyq_layernorm_workspace_bytes", rows, K, C.byref(size)) == EINVAL


def test_norm_of_wide_rows(polyq_lib):
    most = int(re.search(r"POLYQ_NORM_MAX_K (\d+)", open(HEADER).read()).group(1))
    wide = _dense(polyq_lib, stride=1 << 20)
    assert _fwd(polyq_lib, x=wide, y=wide, K=most + 1) == EUNSUPPORTED
    assert _bwd(polyq_lib, x=wide, dy=wide, dx=wide, K=most + 1) == EUNSUPPORTED


def test_norm_arguments(polyq_lib):
    for eps in (-1e-6, NAN, INF):
        assert _fwd(polyq_lib, eps=eps) == EINVAL
    assert _fwd(polyq_lib, stats=A + 4) == EINVAL
    assert _bwd(polyq_lib, stats=None) == EINVAL and _bwd(polyq_lib, stats=A + 4) == EINVAL
    assert _bwd(polyq_lib, dx=None) == EINVAL  # nothing is wanted
    other = _dense(polyq_lib, type=0)
    assert _bwd(polyq_lib, dx=other) == EINVAL and _bwd(polyq_lib, res=other) == EINVAL
    assert _bwd(polyq_lib, dx=None, dw=other, res=_dense(polyq_lib)) == EINVAL


# ---- AdamW ----
def _adam(polyq, tensor=None, n=1, types=(0, 1, 1), state=None, hyper=None, tensors=True, hypers=True):
    t = dict(p=A, grad=A, copy=None, n=1000, at=0, decay=0.1, rate=1.0)
    t.update(tensor or {})
    s = dict(m=A, v=A, m_scales=A, v_scales=A, n=1024, bits=8)
    s.update(state or {})
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, lr_dev=None, step_dev=None, grad_scale=None)
    h.update(hyper or {})
    arr = (polyq.AdamwTensor * 1)(polyq.AdamwTensor(*t.values()))
    return _rc(polyq, "polyq_adamw_step", arr if tensors else None, n, *types, polyq.AdamwState(*s.values()),
               polyq.AdamwHyper(*h.values()) if hypers else None, None)


@pytest.mark.parametrize("bad", [
    dict(p=None), dict(grad=None), dict(p=A + 2), dict(grad=A + 1), dict(copy=A + 1), dict(n=0), dict(n=-1),
    dict(n=1025), dict(n=1 << 62), dict(at=256), dict(at=128), dict(at=-256), dict(at=1 << 62), dict(decay=-0.1),
    dict(decay=NAN), dict(rate=-1.0), dict(rate=INF)])
def test_adamw_bad_tensor(polyq_lib, bad):
    assert _adam(polyq_lib, tensor=bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(m=None), dict(v=None), dict(m=A + 8), dict(v=A + 4), dict(m_scales=None),
                                 dict(v_scales=None), dict(n=1000), dict(n=0), dict(n=-256), dict(bits=16)])
def test_adamw_bad_state(polyq_lib, bad):
    assert _adam(polyq_lib, state=bad) == EINVAL
    s = dict(m=A, v=A, m_scales=A, v_scales=A, n=1024, bits=8)
    s.update(bad)
    s, d = polyq_lib.AdamwState(*s.values()), _dense(polyq_lib)
    assert _rc(polyq_lib, "polyq_adamw_values", s, d, d, None) == EINVAL


@pytest.mark.parametrize("bad", [
    dict(lr=-1.0), dict(lr=NAN), dict(lr=INF), dict(lr=1e300), dict(beta1=-0.1), dict(beta1=1.0), dict(beta1=NAN),
    dict(beta2=1.0), dict(beta2=-1e-9), dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=INF), dict(eps=NAN),
    dict(step=0), dict(step=-3), dict(lr_dev=A + 2), dict(step_dev=A + 4), dict(grad_scale=A + 1)])
def test_adamw_bad_rates(polyq_lib, bad):
    assert _adam(polyq_lib, hyper=bad) == EINVAL


def test_adamw_arguments(polyq_lib):
    for types in ((3, 1, 1), (0, -1, 1)):
        assert _adam(polyq_lib, types=types) == EINVAL
    assert _adam(polyq_lib, types=(0, 1, 5), tensor=dict(copy=A)) == EINVAL
    assert _adam(polyq_lib, n=0) == EINVAL and _adam(polyq_lib, n=-1) == EINVAL
    assert _adam(polyq_lib, tensors=False) == EINVAL and _adam(polyq_lib, hypers=False) == EINVAL
    s = polyq_lib.AdamwState(A, A, A, A, 1024, 8)
    for d in (_dense(polyq_lib, data=A + 1), _dense(polyq_lib, type=4), _dense(polyq_lib, data=None)):
        assert _rc(polyq_lib, "polyq_adamw_values", s, d, None, None) == EINVAL
        assert _rc(polyq_lib, "polyq_adamw_values", s, None, d, None) == EINVAL
    assert _rc(polyq_lib, "polyq_adamw_values", s, None, None, None) == EINVAL
    s32 = polyq_lib.AdamwState(A, A, None, None, 1024, 32)
    assert _rc(polyq_lib, "polyq_adamw_values", s32, _dense(polyq_lib), None, None) == EINVAL


# ---- adapters ----
GOOD = dict(a=A, b=A, a_stride=128, a_next=16 * 128, b_stride=16, b_next=64 * 16, K=128, N=64, n=3, R=16, type=1,
            scales=None, ranks=None)


def _lora(polyq, backward=False, x=None, T=8, ad=None, seg=None, res=None, y="y", saved=A, dy=None, da=A, db=A,
          gt=0, ws=A, n=1 << 40, no=()):
    d = _dense(polyq)
    a = dict(GOOD)
    a.update(ad or {})
    s = dict(offsets=A, ids=A, n=2)
    s.update(seg or {})
    a = None if "adapters" in no else polyq.Adapters(*a.values())
    s = None if "segments" in no else polyq.Segments(*s.values())
    y = d if y == "y" else y
    if backward:
        return _rc(polyq, "polyq_adapters_backward", x or d, T, a, s, saved, dy or d, res, y, da, db, gt, ws, n, None)
    return _rc(polyq, "polyq_adapters_forward", x or d, T, a, s, res, y, saved, ws, n, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad", [
    dict(a=None), dict(b=None), dict(a=A + 8), dict(b=A + 2), dict(a_stride=120), dict(a_stride=132), dict(b_stride=8),
    dict(b_stride=20), dict(a_next=-8), dict(a_next=4), dict(b_next=12), dict(K=0), dict(K=-1), dict(N=0),
    dict(N=(1 << 24) + 1), dict(n=0), dict(n=-1), dict(R=0), dict(R=-8), dict(R=12), dict(type=0), dict(type=7),
    dict(scales=A + 2), dict(ranks=A + 1)])
def test_bad_adapters(polyq_lib, bad, back):
    assert _lora(polyq_lib, back, ad=bad) == EINVAL


@pytest.mark.parametrize("back", [False, True])
def test_adapters_rank_past_the_limit(polyq_lib, back):
    assert _lora(polyq_lib, back, ad=dict(R=136, b_stride=136)) == EUNSUPPORTED


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad", [dict(offsets=None), dict(ids=None), dict(offsets=A + 2), dict(ids=A + 1), dict(n=0),
                                 dict(n=-2)])
def test_bad_segments(polyq_lib, bad, back):
    assert _lora(polyq_lib, back, seg=bad) == EINVAL


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad", BAD + [dict(type=0), dict(type=2)])
def test_adapters_of_a_bad_tensor(polyq_lib, bad, back):
    d = _dense(polyq_lib, **bad)
    assert _lora(polyq_lib, back, x=d) == EINVAL
    if back:
        if bad != dict(stride=127):  # (127 holds the 64 columns of dy)
            assert _lora(polyq_lib, True, dy=d) == EINVAL
        assert _lora(polyq_lib, True, dy=_dense(polyq_lib, stride=60)) == EINVAL
    if bad in BAD[:2] + BAD[4:]:
        assert _lora(polyq_lib, back, y=d) == EINVAL and _lora(polyq_lib, back, res=d) == EINVAL


@pytest.mark.parametrize("back", [False, True])
def test_adapters_arguments(polyq_lib, back):
    for T in (0, -1, (1 << 24) + 1):
        assert _lora(polyq_lib, back, T=T) == EINVAL
    for no in ("adapters", "segments"):
        assert _lora(polyq_lib, back, no=(no,)) == EINVAL
    # an output of neither type, a residual of another one, a residual in place with another stride
    assert _lora(polyq_lib, back, y=_dense(polyq_lib, type=2)) == EINVAL
    assert _lora(polyq_lib, back, res=_dense(polyq_lib, type=0)) == EINVAL
    assert _lora(polyq_lib, back, res=_dense(polyq_lib, stride=256)) == EINVAL
    assert _lora(polyq_lib, back, saved=A + 8) == EINVAL and _lora(polyq_lib, back, ws=A + 8) == EINVAL
    need = C.c_size_t()
    assert polyq_lib._lib.polyq_adapters_workspace_bytes(8, 16, C.byref(need)) == 0 and need.value == 256 + 8 * 16 * 4
    assert _lora(polyq_lib, back, n=need.value - 1) == ENOMEM and _lora(polyq_lib, back, ws=None) == ENOMEM
    for T, R in ((0, 16), (8, 0), (8, 12), (8, 136), ((1 << 24) + 1, 16)):
        assert _rc(polyq_lib, "polyq_adapters_workspace_bytes", T, R, C.byref(need)) == EINVAL
    assert _rc(polyq_lib, "polyq_adapters_workspace_bytes", 8, 16, None) == EINVAL


def test_adapters_gradients(polyq_lib):
    assert _lora(polyq_lib, True, y=None, da=None, db=None) == EINVAL
    assert _lora(polyq_lib, True, saved=None) == EINVAL  # db needs it
    assert _lora(polyq_lib, True, gt=2) == EINVAL and _lora(polyq_lib, True, gt=9) == EINVAL
    assert _lora(polyq_lib, True, da=A + 2) == EINVAL and _lora(polyq_lib, True, db=A + 1) == EINVAL
    assert _lora(polyq_lib, True, y=None, res=_dense(polyq_lib)) == EINVAL


# ---- the binding's own checks ----
def test_binding_refuses_what_is_no_cuda_tensor(polyq_lib):
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    a, b = torch.zeros(1, 8, 16, dtype=torch.bfloat16), torch.zeros(1, 16, 8, dtype=torch.bfloat16)
    off, ids = torch.tensor([0, 4], dtype=torch.int32), torch.tensor([0], dtype=torch.int32)
    state = polyq_lib.AdamState([16], device="cpu")
    for bad in (x, 7, "buffer", None, [1], x.to(torch.int32)):
        for call in (lambda: polyq_lib.layernorm_forward(bad), lambda: polyq_lib.layernorm_backward(bad, None, None, bad),
                     lambda: polyq_lib.adapters_forward(bad, a, b, off, ids),
                     lambda: polyq_lib.adapters_backward(bad, a, b, None, bad, off, ids),
                     lambda: polyq_lib.AdamW([bad], [bad], state)):
            with pytest.raises(ValueError):
                call()


def test_adam_state_arguments(polyq_lib):
    for sizes, bits in (([], 32), ([0], 32), ([5, -1], 8), ([5], 16)):
        with pytest.raises(ValueError):
            polyq_lib.AdamState(sizes, bits, "cpu")
    s = polyq_lib.AdamState([5, 256, 300], 8, "cpu")
    assert s.offsets == (0, 256, 512) and s.m.numel() == 1024 and s.m_scales.numel() == 4
    with pytest.raises(AttributeError):
        s.m = s.v
    with pytest.raises(ValueError):
        s.values()
    with pytest.raises(ValueError):
        polyq_lib.AdamW([], [], s)


@pytest.mark.parametrize("name,pack", [("Dense", "_pack_dense"), ("Adapters", "_pack_adapters"),
                                       ("Segments", "_pack_segments"), ("AdamwHyper", "_pack_hyper")])
def test_packed_descriptors(polyq_lib, name, pack):
    """The bytes that calls pass are those of the structures of the header."""
    import ctypes as C
    kind = getattr(polyq_lib, name)
    values = [(i + 1) * (0.25 if t is C.c_double else 3) for i, (_, t) in enumerate(kind._fields_)]
    assert getattr(polyq_lib, pack)(*values) == bytes(kind(*values))
