"""GPU tests of the 4-bit products and the gated block at sizes that reach every
way a call can be launched, against 64-bit products on the GPU; and of calls
together: captured, replayed, on other streams, one feeding the next."""
import numpy as np
import pytest

from tests.fp4_util import U32, half_step, tiny

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MX, NV = 0, 1


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _q(polyq, g, rows, K, fmt, scale=0.1):
    x = torch.randn(rows, K, generator=g, device="cuda") * scale
    return polyq.fp4_quantize(x, fmt, 1.0 if fmt == MX else 2.0 ** -8)


def _values(polyq, q):
    return polyq.fp4_dequantize(q, torch.float32).double()


def _sum_bound(S, K, per, parts=10):
    # as fp4_util.sum_bound, with the parts that pairs of SMs share counted too
    return (2 * (-(-K // per)) + 10 + parts) * U32 * S


def _check(got, ref, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    off = (got - ref).abs() - bound
    assert float(off.max()) <= 0, f"{what}: {int((off > 0).sum())} of {off.numel()} off, by {float(off.max())}"


# (M, N, K): tokens beyond one tile of mm_few (64 and 128 tokens), whole waves of
# pair tiles, a last wave in even parts, and in shares that do not end with tiles
LINEAR = [(100, 600, 2000), (200, 1024, 2500), (330, 400, 1100), (513, 700, 600), (1000, 400, 300), (1900, 260, 5000),
          (1500, 5200, 300), (2304, 2560, 13824), (2300, 2500, 7000), (7424, 1024, 40000)]


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N,K", LINEAR)
def test_linear_paths(polyq_lib, fmt, M, N, K):
    g = _gen(M + N + K)
    x, w = _q(polyq_lib, g, M, K, fmt), _q(polyq_lib, g, N, K, fmt)
    ws = polyq_lib.fp4_workspace()
    y = polyq_lib.fp4_linear(x, w, workspace=ws)
    again = polyq_lib.fp4_linear(x, w, workspace=ws)
    assert polyq_lib.workspace_status(ws) == 0
    assert int(ws[:polyq_lib.FP4_WORKSPACE_ZERO].max()) == 0  # ready for the next call
    assert torch.equal(y, again)
    xv, wv = _values(polyq_lib, x), _values(polyq_lib, w)
    _check(y, xv @ wv.T, _sum_bound(xv.abs() @ wv.abs().T, K, 64, 100) + 2.0 ** -140, "y")


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,F,K", [(70, 600, 2000), (200, 1024, 2500), (330, 400, 1100), (1000, 400, 300),
                                   (1500, 2600, 300), (2304, 1280, 13824), (2300, 1250, 7000), (7424, 512, 40000)])
def test_ffn_paths(polyq_lib, fmt, M, F, K):
    g = _gen(M + F + K)
    x, a, b = _q(polyq_lib, g, M, K, fmt, 1.0), _q(polyq_lib, g, F, K, fmt, K ** -0.5), _q(polyq_lib, g, F, K, fmt, 0.1)
    ws = polyq_lib.fp4_workspace()
    h = polyq_lib.fp4_ffn(x, a, b, dtype=torch.float32, workspace=ws)
    assert torch.equal(h, polyq_lib.fp4_ffn(x, a, b, dtype=torch.float32, workspace=ws))
    assert polyq_lib.workspace_status(ws) == 0
    assert int(ws[:polyq_lib.FP4_WORKSPACE_ZERO].max()) == 0
    xv, av, bv = (_values(polyq_lib, t) for t in (x, a, b))
    s, u = xv @ av.T, xv @ bv.T
    ea, eu = (_sum_bound(xv.abs() @ v.abs().T, K, 64, 100) for v in (av, bv))
    ref = s / (1 + torch.exp(-s)) * u
    bound = 1.1 * ea * (u.abs() + eu) + s.abs() * eu + ref.abs() * (8 + 1.2 * s.abs()) * U32
    _check(h, ref, bound + 2.0 ** -140, "h")
    for ofmt in (MX, NV):
        q = polyq_lib.Fp4Tensor.empty(M, F, ofmt, 1.0 if ofmt == MX else 0.25)
        polyq_lib.fp4_ffn(x, a, b, h=q, workspace=ws)
        want = polyq_lib.fp4_quantize(h, ofmt, q.tensor_scale)
        for p, r in zip(q.unpack(), want.unpack()):
            assert torch.equal(p, r)


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,F,K", [(70, 600, 256), (301, 2731, 1000), (1300, 500, 264), (2304, 5000, 2560),
                                   (6000, 1200, 2304), (1500, 2600, 304)])
def test_training_paths(polyq_lib, t, T, F, K):
    g = _gen(T + F + K)
    x = torch.randn(T, K, generator=g, device="cuda").to(t)
    gate, up = ((torch.randn(F, K, generator=g, device="cuda") / K ** 0.5).to(t) for _ in range(2))
    dh = torch.randn(T, F, generator=g, device="cuda").to(t)
    ws = polyq_lib.ffn_workspace(T, F)
    saved = polyq_lib.ffn_saved(T, F)
    h = polyq_lib.ffn_forward(x, gate, up, saved=saved, workspace=ws)
    X, G, U, D = (v.double() for v in (x, gate, up, dh))
    a, u = X @ G.T, X @ U.T
    ea, eu = (_sum_bound(X.abs() @ v.abs().T, K, 16, 100) for v in (G, U))
    s = 1 / (1 + torch.exp(-a))
    ref = a * s * u
    bound = 1.1 * ea * (u.abs() + eu) + a.abs() * eu + ref.abs() * (8 + 1.2 * a.abs()) * U32
    _check(h, ref, bound * 1.01 + ref.abs() * half_step(t) + tiny(t), "h")
    out = [torch.empty(r, K, device="cuda") for r in (T, F, F)]
    polyq_lib.ffn_backward(x, gate, up, saved, dh, *out, workspace=ws)
    again = [torch.empty_like(o) for o in out]
    polyq_lib.ffn_backward(x, gate, up, saved, dh, *again, workspace=ws)
    assert all(torch.equal(p, q) for p, q in zip(out, again))
    assert polyq_lib.workspace_status(ws) == 0
    # a and u are saved to 2^-15, da and du computed to (12 + 1.2 |a|) units and
    # rounded to half a step of the type; |d(silu)/da| < 1.1, |d2(silu)/da2| <= 1/2
    da, du = D * u * s * (1 + a * (1 - s)), D * a * s
    ea, eu = ea + a.abs() * 2.0 ** -15, eu + u.abs() * 2.0 ** -15
    fa = 1.1 * D.abs() * eu + 0.5 * (D * u).abs() * ea + (D * u).abs() * s * (1 + a.abs()) * (12 + 1.2 * a.abs()) * U32
    fu = 1.1 * D.abs() * ea + du.abs() * (12 + 1.2 * a.abs()) * U32
    fa, fu = (e * 1.02 + v.abs() * half_step(t) * 1.01 + tiny(t) for e, v in ((fa, da), (fu, du)))
    refs = [(da @ G + du @ U, fa @ G.abs() + fu @ U.abs() +
             _sum_bound(da.abs() @ G.abs() + du.abs() @ U.abs(), 2 * F, 16, 100)),
            (da.T @ X, fa.T @ X.abs() + _sum_bound(da.abs().T @ X.abs(), T, 16, 100)),
            (du.T @ X, fu.T @ X.abs() + _sum_bound(du.abs().T @ X.abs(), T, 16, 100))]
    for n, o, (r, e) in zip(("dx", "dgate", "dup"), out, refs):
        _check(o, r, e * 1.02 + 2.0 ** -140, n)


def _block(polyq, M, K, F, fmt, seed):
    """The quantised block of a decoder layer: operands, and a call that runs it."""
    g = _gen(seed)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    gate, up = (_q(polyq, g, F, K, fmt, K ** -0.5) for _ in range(2))
    down = _q(polyq, g, K, F, fmt, F ** -0.5)
    res = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    ts = 1.0 if fmt == MX else 2.0 ** -6
    xq, hq = polyq.Fp4Tensor.empty(M, K, fmt, ts), polyq.Fp4Tensor.empty(M, F, fmt, ts)
    y, ws = torch.empty_like(res), polyq.fp4_workspace()

    def run(stream=None):
        polyq.fp4_quantize(x, out=xq, stream=stream)
        polyq.fp4_ffn(xq, gate, up, hq, workspace=ws, stream=stream)
        polyq.fp4_linear(hq, down, y=y, residual=res, workspace=ws, stream=stream)
        return y

    return x, (xq, hq, gate, up, down, res, ws), run


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,K,F", [(1, 512, 1408), (37, 264, 777), (300, 1000, 1111), (2500, 512, 2600)])
def test_block_together(polyq_lib, fmt, M, K, F):
    """Activations quantised, gate and up with a quantised output, down with the
    residual: each call's result is the product of what the calls before wrote."""
    x, (xq, hq, gate, up, down, res, ws), run = _block(polyq_lib, M, K, F, fmt, M)
    y = run()
    want = polyq_lib.fp4_quantize(x, fmt, xq.tensor_scale)
    assert all(torch.equal(p, q) for p, q in zip(xq.unpack(), want.unpack()))
    xv, av, bv, hv, dv = (_values(polyq_lib, t) for t in (xq, gate, up, hq, down))
    h = polyq_lib.fp4_ffn(xq, gate, up, dtype=torch.float32)
    want = polyq_lib.fp4_quantize(h, fmt, hq.tensor_scale)
    assert all(torch.equal(p, q) for p, q in zip(hq.unpack(), want.unpack()))
    s = xv @ av.T
    ref = s / (1 + torch.exp(-s)) * (xv @ bv.T)
    assert float((h.double() - ref).norm() / ref.norm()) < 1e-5
    ref = res.double() + hv @ dv.T
    S = res.double().abs() + hv.abs() @ dv.abs().T
    _check(y, ref, _sum_bound(S, F, 64, 100) * 1.01 + ref.abs() * half_step(torch.bfloat16) + 2.0 ** -140, "y")


@pytest.mark.parametrize("M", [1, 300, 2304])
def test_captured_and_replayed(polyq_lib, M):
    """The block in a CUDA graph, replayed on new inputs, twice in one graph."""
    x, _, run = _block(polyq_lib, M, 512, 1408, MX, 7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
        y = run()
    for seed in (1, 2):
        x.copy_(torch.randn(x.shape, generator=_gen(seed), device="cuda").bfloat16())
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, run())


def test_short_calls_over_the_same_buffers(polyq_lib):
    """Launches that overlap in a graph read what the one before them wrote, not
    what the buffer held in an earlier call."""
    n, T, F, K = 40, 8, 96, 64
    g = _gen(11)
    x = torch.randn(n, T, K, generator=g, device="cuda").bfloat16()
    gate, up = (torch.randn(F, K, generator=g, device="cuda").bfloat16() for _ in range(2))
    dh = torch.randn(T, F, generator=g, device="cuda").bfloat16()
    w = _q(polyq_lib, g, 200, F, MX)
    ws = polyq_lib.ffn_workspace(T, F)

    def buffers():
        return (torch.empty(T, F, dtype=torch.bfloat16, device="cuda"), polyq_lib.ffn_saved(T, F),
                polyq_lib.Fp4Tensor.empty(T, F, MX), torch.empty(T, F, device="cuda"))

    def run(x, h, saved, q, v, y, dx):
        polyq_lib.ffn_forward(x, gate, up, h=h, saved=saved, workspace=ws)
        polyq_lib.fp4_quantize(h, out=q)
        polyq_lib.fp4_dequantize(q, out=v)
        polyq_lib.fp4_linear(q, w, y=y, workspace=ws)
        polyq_lib.ffn_backward(x, gate, up, saved, dh, dx=dx, need_weights=False, workspace=ws)
        polyq_lib.fp4_quantize(v, out=q)

    def outs():
        return torch.empty(n, T, 200, device="cuda"), torch.empty(n, T, K, dtype=torch.bfloat16, device="cuda")

    (y, dx), (y1, dx1) = outs(), outs()
    for i in range(n):
        run(x[i], *buffers(), y1[i], dx1[i])
        torch.cuda.synchronize()
    shared = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(n):
            run(x[i], *shared, y[i], dx[i])
    for _ in range(3):
        y.fill_(float("nan"))
        dx.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y1) and torch.equal(dx, dx1)


def test_streams_with_their_own_workspaces(polyq_lib):
    """Two blocks at once on two streams, each with its buffers, give what they
    give alone; a given stream is used although another is current."""
    blocks = [_block(polyq_lib, M, 512, 1408, f, M) for M, f in ((300, MX), (2304, NV))]
    alone = [b[2]().clone() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        outs = [b[2](stream=s) for b, s in zip(blocks, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(alone, outs))


def test_buffers_made_for_a_given_stream(polyq_lib):
    """Without buffers of the caller's, on a stream that is not the current one,
    while the current one is busy: the new workspace is zeroed on that stream."""
    g = _gen(4)
    x, w = _q(polyq_lib, g, 2304, 7000, MX), _q(polyq_lib, g, 2560, 7000, MX)  # shares its last wave
    h = torch.randn(300, 512, generator=g, device="cuda").bfloat16()
    want = (polyq_lib.fp4_linear(x, w), polyq_lib.fp4_ffn(x, w, w), polyq_lib.ffn_forward(h, h, h))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        junk = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")  # what new memory may hold
        del junk
        torch.cuda._sleep(20_000_000)
        got = (polyq_lib.fp4_linear(x, w, stream=side), polyq_lib.fp4_ffn(x, w, w, stream=side),
               polyq_lib.ffn_forward(h, h, h, stream=side))
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()


def test_training_step_captured(polyq_lib):
    """Forward and backward in a CUDA graph, replayed after the inputs changed."""
    T, F, K, t = 300, 264, 136, torch.bfloat16
    x, gate, up = (torch.randn(r, K, device="cuda").to(t) for r in (T, F, F))
    dh = torch.randn(T, F, device="cuda").to(t)
    saved, ws = polyq_lib.ffn_saved(T, F), polyq_lib.ffn_workspace(T, F)
    h, grads = torch.empty_like(dh), [torch.empty_like(v) for v in (x, gate, up)]

    def step():
        polyq_lib.ffn_forward(x, gate, up, h=h, saved=saved, workspace=ws)
        polyq_lib.ffn_backward(x, gate, up, saved, dh, *grads, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (3, 4):
        for v in (x, dh):
            v.copy_(torch.randn(v.shape, generator=_gen(seed), device="cuda").to(t))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (h, *grads)]
        step()
        assert all(torch.equal(p, q) for p, q in zip(got, (h, *grads)))


def test_fake_quantised_weights_train_what_is_served(polyq_lib):
    """A training step on fake-quantised weights and activations and the served
    block on the quantised ones multiply the same numbers (bf16 holds every e2m1
    multiple of an e8m0 scale): their fp32 sums differ by rounding only."""
    g = _gen(5)
    M, F, K = 200, 300, 512
    q = [polyq_lib.fp4_quantize(torch.randn(r, K, generator=g, device="cuda") * s, MX)
         for r, s in ((M, 1.0), (F, K ** -0.5), (F, K ** -0.5))]
    fake = [polyq_lib.fp4_dequantize(t, torch.bfloat16) for t in q]
    assert all(torch.equal(f.double(), _values(polyq_lib, t)) for f, t in zip(fake, q))
    trained = polyq_lib.ffn_forward(*fake)
    served = polyq_lib.fp4_ffn(*q, dtype=torch.bfloat16)
    v = [f.double() for f in fake]
    a, u = v[0] @ v[1].T, v[0] @ v[2].T
    ref = a / (1 + torch.exp(-a)) * u
    S = [v[0].abs() @ w.abs().T for w in v[1:]]
    ea, eu = (_sum_bound(s, K, 16) for s in S)
    bound = 1.1 * ea * (u.abs() + eu) + a.abs() * eu + ref.abs() * (8 + 1.2 * a.abs()) * U32
    for h in (trained, served):
        _check(h, ref, bound * 1.01 + ref.abs() * half_step(torch.bfloat16) + 2.0 ** -133, "h")


def test_offsets_beyond_32_bits(polyq_lib):
    """Tensors of more than 2^32 elements: their last rows are what a small call gives."""
    rows, K = 300000, 16384
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    x[:300].normal_(generator=_gen(1))
    x[-300:].normal_(generator=_gen(2))
    x[300:-300].zero_()
    for fmt in (MX, NV):
        q = polyq_lib.fp4_quantize(x, fmt)
        last = polyq_lib.fp4_quantize(x[-300:].contiguous(), fmt)
        v = polyq_lib.fp4_dequantize(q, torch.bfloat16)
        assert torch.equal(v[-300:], polyq_lib.fp4_dequantize(last, torch.bfloat16))
        assert torch.equal(v[:300], polyq_lib.fp4_dequantize(polyq_lib.fp4_quantize(x[:300], fmt), torch.bfloat16))
        assert not bool(v[300:-300].any())
    del x, v
    # an output of more than 2^32 elements, from rows whose codes are far into theirs
    w = _q(polyq_lib, _gen(3), 16640, K, NV)
    y = polyq_lib.fp4_linear(q, w, dtype=torch.bfloat16)
    part = polyq_lib.fp4_linear(last, w, dtype=torch.bfloat16)
    assert float((y[-300:].double() - part.double()).norm() / part.double().norm()) < 4e-3
    assert not bool(y[300:-300].any())


@pytest.mark.parametrize("fmt", [MX, NV])
def test_code_rows_of_a_wider_buffer(polyq_lib, fmt):
    """Codes with a stride of their own: what lies behind a row does not matter."""
    import ctypes as C
    g = _gen(9)
    M, N, K = 150, 140, 333
    x, w = _q(polyq_lib, g, M, K, fmt), _q(polyq_lib, g, N, K, fmt)
    y = polyq_lib.fp4_linear(x, w)
    buffers = []
    for t in (x, w):
        wide = torch.full((t.rows, 512), 0x77, dtype=torch.uint8, device="cuda")
        wide[:, :t.codes.shape[1]] = t.codes
        wide[:, (K + 1) // 2:] = 0x77  # also the padding of the narrow rows
        t.desc.codes, t.desc.code_stride = wide.data_ptr(), 512
        buffers.append(wide)
    assert torch.equal(y, polyq_lib.fp4_linear(x, w))
    src = torch.randn(M, K, generator=g, device="cuda")
    d = polyq_lib._dense(src, "x")
    rc = polyq_lib._lib.polyq_fp4_quantize(C.byref(d), C.byref(x.desc), polyq_lib._stream_ptr(None))
    assert rc == 0
    want = polyq_lib.fp4_quantize(src, fmt, x.tensor_scale)
    got = buffers[0]
    assert torch.equal(got[:, :(K + 1) // 2], want.codes[:, :(K + 1) // 2])
    assert bool((got[:, 176:] == 0x77).all())  # 16-byte rows: 176 bytes of 333 codes


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N", [(1, 8), (40, 130), (300, 257)])
def test_long_contraction(polyq_lib, fmt, M, N):
    """A million products a sum."""
    K = (1 << 20) + 37
    g = _gen(M)
    x, w = _q(polyq_lib, g, M, K, fmt), _q(polyq_lib, g, N, K, fmt)
    xv, wv = _values(polyq_lib, x), _values(polyq_lib, w)
    ref, S = xv @ wv.T, xv.abs() @ wv.abs().T
    _check(polyq_lib.fp4_linear(x, w), ref, _sum_bound(S, K, 64, 100), "y")
    assert float((polyq_lib.fp4_linear(x, w).double() - ref).norm() / ref.norm()) < 1e-3


def test_python_refusals_on_the_gpu(polyq_lib):
    x = torch.randn(8, 64, device="cuda")
    q = polyq_lib.fp4_quantize(x)
    h = x.bfloat16()
    ws, fws = polyq_lib.fp4_workspace(), polyq_lib.ffn_workspace(8, 8)
    saved = polyq_lib.ffn_saved(8, 8)
    bad = [
        lambda: polyq_lib.fp4_quantize(x.double()), lambda: polyq_lib.fp4_quantize(x[0]),
        lambda: polyq_lib.fp4_quantize(x.T), lambda: polyq_lib.fp4_quantize(x[:1].expand(8, 64)),
        lambda: polyq_lib.fp4_quantize(x[:4], out=q), lambda: polyq_lib.fp4_dequantize(q, out=x[:4]),
        lambda: polyq_lib.fp4_linear(q, q, y=torch.empty(8, 9, device="cuda")),
        lambda: polyq_lib.fp4_linear(q, q, y=torch.empty(8, 8)),
        lambda: polyq_lib.fp4_linear(q, q, residual=torch.empty(8, 7, device="cuda")),
        lambda: polyq_lib.fp4_linear(q, q, workspace=ws[:256].float()),
        lambda: polyq_lib.fp4_ffn(q, q, x),
        lambda: polyq_lib.ffn_forward(h, h, x), lambda: polyq_lib.ffn_forward(h, h[:, :32], h[:, :32]),
        lambda: polyq_lib.ffn_forward(h, h, h, saved=saved[:-6]),
        lambda: polyq_lib.ffn_backward(h, h, h, saved, x[:, :8]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {i} was not refused")
    refused = [
        lambda: polyq_lib.ffn_forward(x, x, x), lambda: polyq_lib.fp4_linear(q, q, workspace=ws[:-256]),
        lambda: polyq_lib.fp4_linear(q, polyq_lib.fp4_quantize(x, NV)),
        lambda: polyq_lib.fp4_linear(q, polyq_lib.fp4_quantize(x[:, :32])),
        lambda: polyq_lib.fp4_ffn(q, q, q, polyq_lib.Fp4Tensor.empty(8, 9)),
        lambda: polyq_lib.ffn_forward(h[:, 1:], h[:, 1:], h[:, 1:]),
        lambda: polyq_lib.ffn_backward(h, h, h, saved, h[:, :8], workspace=fws[:-256]),
        lambda: polyq_lib.fp4_quantize(x, NV, 0.0), lambda: polyq_lib.fp4_quantize(x, MX, 2.0),
        lambda: polyq_lib.fp4_quantize(x, 7),
    ]
    for call in refused:
        with pytest.raises(polyq_lib.PolyqError):
            call()
    assert polyq_lib.workspace_status(ws) == 0
