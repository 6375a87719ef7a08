"""GPU tests of layer norm, 4-bit products, adapters and AdamW together, as a fine-tuning step
of a quantised projection and the serving of its result use them; and of large tensors, calls at
once and arguments."""
import numpy as np
import pytest
import torch

from tests import finetune_util as F
from tests.test_gpu_adapters import make, segments, within

pytestmark = pytest.mark.gpu


class Step:
    """A norm, a projection with 4-bit weights and two adapters, all on fixed buffers."""

    def __init__(self, polyq, bits, T=300, K=512, N=640, R=16, seed=0):
        self.polyq = polyq
        g = torch.Generator("cuda").manual_seed(seed)

        def rnd(*s):
            return torch.randn(*s, generator=g, device="cuda")

        self.x, self.dy = rnd(T, K).bfloat16(), rnd(T, N).bfloat16()
        self.gain = 1 + 0.1 * rnd(K)
        self.a, self.b = rnd(2, R, K) * K ** -0.5, 0.1 * rnd(2, N, R)
        self.a16, self.b16 = self.a.bfloat16(), self.b.bfloat16()
        self.w = polyq.fp4_quantize((rnd(N, K) * K ** -0.5).bfloat16())
        self.w_dense = polyq.fp4_dequantize(self.w)
        self.off = torch.tensor([0, 100, 250, T], dtype=torch.int32, device="cuda")
        self.ids = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
        self.scales = torch.tensor([2.0, 0.5], device="cuda")
        self.grads = [torch.zeros_like(t) for t in (self.gain, self.a, self.b)]
        self.state = polyq.AdamState([K, 2 * R * K, 2 * N * R], bits)
        self.plan = polyq.AdamW([self.gain, self.a, self.b], self.grads, self.state,
                                copies=[None, self.a16, self.b16], weight_decay=[0.0, 0.1, 0.1])
        self.ws, self.ws4 = polyq.adapters_workspace(T, R), polyq.fp4_workspace()
        self.wsn, self.stats = polyq.layernorm_workspace(T, K), polyq.layernorm_stats(T)
        self.saved = polyq.adapters_saved(T, R)
        self.count = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.h, self.dh, self.dx = (torch.empty_like(self.x) for _ in range(3))
        self.y = torch.empty_like(self.dy)
        self.xq = polyq.Fp4Tensor.empty(T, K)

    def forward(self):
        p = self.polyq
        p.layernorm_forward(self.x, self.gain, center=False, y=self.h, stats=self.stats)
        p.fp4_quantize(self.h, out=self.xq)
        p.fp4_linear(self.xq, self.w, y=self.y, workspace=self.ws4)
        return p.adapters_forward(self.h, self.a16, self.b16, self.off, self.ids, scales=self.scales, residual=self.y,
                                  y=self.y, saved=self.saved, workspace=self.ws)

    def backward(self):
        p = self.polyq
        # the projection's own part, straight through the quantiser of its input
        torch.mm(self.dy, self.w_dense.bfloat16(), out=self.dh)
        p.adapters_backward(self.h, self.a16, self.b16, self.saved, self.dy, self.off, self.ids, scales=self.scales,
                            residual=self.dh, dx=self.dh, da=self.grads[1], db=self.grads[2], workspace=self.ws)
        p.layernorm_backward(self.x, self.gain, self.stats, self.dh, center=False, dx=self.dx, dweight=self.grads[0],
                             need_bias=False, workspace=self.wsn)

    def update(self):
        self.count.add_(1)
        self.plan.step(1e-2, self.count, seed=17)

    def run(self):
        self.forward()
        self.backward()
        self.update()

    def results(self):
        return [self.y, self.dx, *self.grads, self.gain, self.a, self.b, self.a16, self.b16, self.state.m, self.state.v]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_fine_tuning_step(polyq_lib, bits):
    s = Step(polyq_lib, bits)
    before = [t.clone() for t in (s.gain, s.a, s.b)]
    leaves = [t.double().requires_grad_() for t in (s.x, s.gain, s.a16, s.b16)]
    s.forward()
    s.backward()
    x, gain, a, b = leaves
    h = x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5) * gain
    base = polyq_lib.fp4_dequantize(s.xq).double() + (h - h.detach())
    y = base @ s.w_dense.double().T
    for s0, s1, i in ((0, 100, 1), (100, 250, 0), (250, 300, 1)):
        y = y + torch.nn.functional.pad(float(s.scales[i]) * (h[s0:s1] @ a[i].T) @ b[i].T, (0, 0, s0, 300 - s1))
    (y * s.dy.double()).sum().backward()
    # at most eight roundings to bf16 (2^-9 each) lie between the inputs and any of these
    for got, ref, what in ((s.y, y.detach(), "y"), (s.dx, x.grad, "dx"), (s.grads[0], gain.grad, "dgain"),
                           (s.grads[1], a.grad, "da"), (s.grads[2], b.grad, "db")):
        assert (got.double() - ref).norm() <= 8 * 2.0 ** -9 * ref.norm(), what
    s.update()
    for p, old, g, decay in zip((s.gain, s.a, s.b), before, s.grads, (0.0, 0.1, 0.1)):
        old, g = (t.double().cpu().numpy().ravel() for t in (old, g))
        ref, m, v, upd = F.adamw(old, g, 0 * g, 0 * g, 1, 1e-2, 0.9, 0.999, 1e-8, decay)
        bound = F.adamw_bounds(old, g, 0 * g, 0 * g, upd, ref, m, v, 0.9, 0.999, 1e-2, decay, torch.float32)[0]
        # (the corrections 1 - beta^t from the device's step: four units of fp32 more)
        assert (np.abs(p.double().cpu().numpy().ravel() - ref) <= bound + 4 * F.U32 * np.abs(upd)).all()
    assert torch.equal(s.a16, s.a.bfloat16()) and torch.equal(s.b16, s.b.bfloat16())
    # served afterwards: a request of one token with the trained adapter
    ids = torch.tensor([1], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    one = polyq_lib.adapters_forward(s.h[:1], s.a16, s.b16, off, ids, scales=s.scales, dtype=torch.float32)
    zero = torch.zeros(1, 640, dtype=torch.float64, device="cuda")
    ref = F.adapters(s.h[:1], s.a16, s.b16, [0, 1], [1], s.scales.tolist(), [16, 16], zero, out=torch.float32)
    within(one, *ref[0], "one token")


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_equal_eager_ones(polyq_lib, bits):
    a, b = Step(polyq_lib, bits), Step(polyq_lib, bits)
    a.run()  # (the library's first use on a stream is not captured)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.run()
    for _ in range(3):
        graph.replay()
    for _ in range(4):
        b.run()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(a.results(), b.results()))
    assert polyq_lib.workspace_status(a.ws) == 0 and polyq_lib.workspace_status(b.ws) == 0


def test_calls_at_once(polyq_lib):
    """Two streams, each with its own buffers, give what one after the other gives."""
    steps = [Step(polyq_lib, 8, seed=i) for i in range(2)]
    twins = [Step(polyq_lib, 8, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for t in twins:
        for _ in range(3):
            t.run()
    torch.cuda.synchronize()
    for s, t in zip(steps, twins):
        assert all(torch.equal(p, q) for p, q in zip(s.results(), t.results()))


def test_offsets_past_32_bits(polyq_lib):
    """Rows, adapters and parameters that begin behind the first 2^32 bytes and 2^31 elements."""
    stride = (1 << 30) + 8
    buf = torch.empty(2 * stride + 640, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 640), (stride, 1))
    x.copy_(torch.randn(3, 640, device="cuda"))
    y = polyq_lib.layernorm_forward(x)
    assert torch.equal(y, polyq_lib.layernorm_forward(x.contiguous()))
    n, R, K, N = 530, 16, 64, 128
    a = torch.empty(n * (1 << 22), dtype=torch.bfloat16, device="cuda").as_strided((n, R, K), (1 << 22, K, 1))
    b = torch.zeros(n, N, R, dtype=torch.bfloat16, device="cuda")
    for i in (0, n - 1):
        a[i].copy_(torch.randn(R, K, device="cuda"))
        b[i].copy_(torch.randn(N, R, device="cuda"))
    for T in (4, 200):
        z = torch.randn(T, K, device="cuda").bfloat16()
        off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
        got = polyq_lib.adapters_forward(z, a, b, off, torch.tensor([n - 1], dtype=torch.int32, device="cuda"))
        want = polyq_lib.adapters_forward(z, a[n - 1:].contiguous(), b[n - 1:].contiguous(), off,
                                          torch.tensor([0], dtype=torch.int32, device="cuda"))
        assert torch.equal(got, want)
    del a, buf, x


def test_a_parameter_of_more_than_2_31_elements(polyq_lib):
    n = (1 << 31) + 1000
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    p[-600:], g[-600:] = torch.randn(600, device="cuda"), torch.randn(600, device="cuda")
    q, h = p[-1000:].clone(), g[-1000:].clone()
    s, t = polyq_lib.AdamState([n], 8), polyq_lib.AdamState([1000], 8)
    polyq_lib.AdamW([p], [g], s).step(0.1, 1)
    polyq_lib.AdamW([q], [h], t).step(0.1, 1)
    assert torch.equal(p[-1000:], q) and not p[:1000].any()
    assert s.m_scales[-3:].any() and not s.m[:1 << 20].any()


BAD = [7, "buffer", [1], object()]


@pytest.mark.parametrize("bad", BAD, ids=[type(b).__name__ for b in BAD])
def test_no_tensor_for_a_buffer(polyq_lib, bad):
    x, a, b, dy, _, _ = make(4, 64, 32, 8, 1, torch.bfloat16)
    off = segments([4])[1]
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    saved, stats = polyq_lib.adapters_saved(4, 8), polyq_lib.layernorm_stats(4)
    p = [torch.zeros(8, device="cuda")]
    state = polyq_lib.AdamState([8])
    plan = polyq_lib.AdamW(p, p, state)
    fwd = polyq_lib.adapters_forward
    for call in (lambda: polyq_lib.layernorm_forward(x, bad), lambda: polyq_lib.layernorm_forward(x, None, bad),
                 lambda: polyq_lib.layernorm_forward(x, y=bad), lambda: polyq_lib.layernorm_forward(x, stats=bad),
                 lambda: polyq_lib.layernorm_backward(x, None, bad, x), lambda: polyq_lib.layernorm_backward(x, None, stats, bad),
                 lambda: polyq_lib.layernorm_backward(x, None, stats, x, workspace=bad),
                 lambda: polyq_lib.layernorm_backward(x, None, stats, x, dweight=bad),
                 lambda: fwd(x, bad, b, off, ids), lambda: fwd(x, a, bad, off, ids), lambda: fwd(x, a, b, bad, ids),
                 lambda: fwd(x, a, b, off, bad), lambda: fwd(x, a, b, off, ids, scales=bad),
                 lambda: fwd(x, a, b, off, ids, ranks=bad), lambda: fwd(x, a, b, off, ids, residual=bad),
                 lambda: fwd(x, a, b, off, ids, saved=bad), lambda: fwd(x, a, b, off, ids, workspace=bad),
                 lambda: polyq_lib.adapters_backward(x, a, b, bad, dy, off, ids),
                 lambda: polyq_lib.adapters_backward(x, a, b, saved, dy, off, ids, da=bad),
                 lambda: polyq_lib.adapters_backward(x, a, b, saved, dy, off, ids, dx=bad),
                 lambda: polyq_lib.AdamW(bad if isinstance(bad, list) else [bad], p, state),
                 lambda: polyq_lib.AdamW(p, p, bad), lambda: plan.step(1e-3, 1, grad_scale=bad)):
        with pytest.raises(ValueError):
            call()


def test_tensors_that_do_not_fit(polyq_lib):
    x, a, b, dy, _, _ = make(6, 64, 32, 8, 2, torch.bfloat16)
    off = segments([4, 2])[1]
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    fwd = polyq_lib.adapters_forward
    i64 = off.long()
    for call in (lambda: fwd(x, a[:1], b, off, ids), lambda: fwd(x, a, b[:, :, :4], off, ids),
                 lambda: fwd(x, a.half(), b, off, ids), lambda: fwd(x.float(), a.float(), b.float(), off, ids),
                 lambda: fwd(x, a, b, i64, ids), lambda: fwd(x, a, b, off[:2], ids), lambda: fwd(x, a, b, off, off),
                 lambda: fwd(x, a, b, off.cpu(), ids), lambda: fwd(x, a, b, off, ids, scales=torch.ones(3, device="cuda")),
                 lambda: fwd(x, a, b, off, ids, residual=dy[:5]),
                 lambda: fwd(x, a, b, off, ids, saved=polyq_lib.adapters_saved(5, 8)),
                 lambda: fwd(x, a.transpose(1, 2), b, off, ids),
                 lambda: polyq_lib.layernorm_forward(x, torch.ones(63, device="cuda")),
                 lambda: polyq_lib.layernorm_forward(x, torch.ones(128, device="cuda")[::2]),
                 lambda: polyq_lib.AdamW([x.t()], [x.t()], polyq_lib.AdamState([384])),
                 lambda: polyq_lib.AdamW([x], [x], polyq_lib.AdamState([383]))):
        with pytest.raises(ValueError):
            call()
    # alignment, types of outputs, workspaces: the library's own checks
    wide = torch.zeros(6, 72, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: fwd(x, wide[None, :2, 1:65].expand(2, 2, 64), b[:, :, :2], off, ids),
                 lambda: fwd(x, a, b, off, ids, dtype=torch.float16),
                 lambda: fwd(x, a, b, off, ids, workspace=torch.zeros(300, dtype=torch.uint8, device="cuda")),
                 lambda: fwd(x[:0], a, b, off, ids), lambda: fwd(x, a, b, off[:1], ids[:0])):
        with pytest.raises(polyq_lib.PolyqError):
            call()
    with pytest.raises(polyq_lib.PolyqError):
        polyq_lib.AdamW([x.clone()], [x], polyq_lib.AdamState([384])).step(1e-3, 0)
    with pytest.raises(polyq_lib.PolyqError):
        polyq_lib.layernorm_forward(torch.zeros(1, 24577, device="cuda"))
