"""GPU tests of the AdamW step over many tensors, with states in 32 and in 8 bits."""
import numpy as np
import pytest
import torch

from tests import finetune_util as F
from tests.fp4_util import check, f64

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LR, B1, B2, EPS = 1e-3, 0.9, 0.95, 1e-8


def tensors(sizes, tp, tg, seed=0, offset=0, copy=None):
    r = np.random.default_rng(seed)

    def put(v, t):
        buf = torch.zeros(len(v) + offset, dtype=t, device="cuda")
        buf[offset:] = torch.from_numpy(v)
        return buf[offset:]

    p = [put(0.05 * r.standard_normal(n), tp) for n in sizes]
    g = [put(1e-2 * r.standard_normal(n), tg) for n in sizes]
    c = None if copy is None else [put(np.full(n, np.nan), copy) for n in sizes]
    return p, g, c


def random_state(polyq, sizes, bits, seed=1):
    """A state in the middle of a run, and its moments per tensor in 64 bits (m, v)."""
    r = np.random.default_rng(seed)
    s = polyq.AdamState(sizes, bits)
    n = s.m.numel()
    if bits == 32:
        m, v = 1e-3 * r.standard_normal(n), (1e-2 * r.standard_normal(n)) ** 2
        s.m.copy_(torch.from_numpy(m))
        s.v.copy_(torch.from_numpy(v))
        m, v = f64(s.m), f64(s.v)
    else:
        cm, cv = r.integers(0, 256, n, dtype=np.uint8), r.integers(1, 256, n, dtype=np.uint8)
        sm, sv = (r.integers(96, 106, n // 256, dtype=np.uint8) for _ in range(2))
        for t, a in ((s.m, cm), (s.v, cv), (s.m_scales, sm), (s.v_scales, sv)):
            t.copy_(torch.from_numpy(a))
        m, v = F.decode(cm, sm, 3, True).ravel(), F.decode(cv, sv, 4, False).ravel() ** 2
    return s, [(m[o:o + k], v[o:o + k]) for o, k in zip(s.offsets, sizes)]


def run(polyq, sizes, tp, tg, bits, copy=None, offset=0, decay=0.1, rate=1.0, t=7, seed=5, scale=None):
    p, g, c = tensors(sizes, tp, tg, offset=offset, copy=copy)
    p0, gs = [f64(x) for x in p], 1.0 if scale is None else float(scale)
    s, before = random_state(polyq, sizes, bits)
    plan = polyq.AdamW(p, g, s, copies=c, weight_decay=decay, lr_scale=rate)
    plan.step(LR, t, betas=(B1, B2), eps=EPS, seed=seed, grad_scale=scale)
    decays = [decay] * len(sizes) if isinstance(decay, float) else decay
    rates = [rate] * len(sizes) if isinstance(rate, float) else rate
    if bits == 8:
        values = [f64(x) for x in s.values()]
        codes = [x.cpu().numpy() for x in (s.m, s.v, s.m_scales, s.v_scales)]
        assert np.array_equal(values[0].reshape(-1, 256), F.decode(codes[0], codes[2], 3, True))
        assert np.array_equal(values[1].reshape(-1, 256), F.decode(codes[1], codes[3], 4, False))
    for i, n in enumerate(sizes):
        grad, (m0, v0), lr = f64(g[i]) * gs, before[i], LR * rates[i]
        ref, m, v, upd = F.adamw(p0[i], grad, m0, v0, t, lr, B1, B2, EPS, decays[i])
        e_p, e_m, e_v = F.adamw_bounds(p0[i], grad, m0, v0, upd, ref, m, v, B1, B2, lr, decays[i], tp)
        check(f64(p[i]), ref, e_p, f"p[{i}]")
        if c is not None:
            assert torch.equal(c[i], p[i].to(copy))
        o = s.offsets[i]
        if bits == 32:
            check(f64(s.m)[o:o + n], m, e_m, f"m[{i}]")
            check(f64(s.v)[o:o + n], v, e_v, f"v[{i}]")
            continue
        blocks = -(-n // 256)
        bits32 = F.noise(seed, o // 256, blocks)

        def wide(a):
            return np.pad(a, (0, blocks * 256 - n)).reshape(blocks, 256)

        for what, a, err, u, mant, got, scales in (
                ("m", np.abs(m), e_m, bits32 & np.uint64(0xFFFF), 3, np.abs(values[0]), codes[2]),
                ("root", np.sqrt(v), 5 * F.U * np.sqrt(v), bits32 >> np.uint64(16), 4, values[1], codes[3])):
            lo, hi, least = F.rounded(wide(a), u.astype(float), mant, wide(err), scales[o // 256:o // 256 + blocks])
            if what == "root":
                lo, hi = (np.where(wide(a) > 0, np.maximum(x, least), x) for x in (lo, hi))
            got = got[o:o + blocks * 256].reshape(blocks, 256)
            bad = (got < lo) | (got > hi)
            assert not bad.any(), (what, i, np.argwhere(bad)[:3])
            assert (lo == hi).mean() > 0.99
        same = np.sign(values[0][o:o + n]) * np.sign(m)
        assert (same >= 0).all() or (np.abs(m[same < 0]) <= e_m[same < 0]).all()
    return p, s


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("tp,tg", [(a, b) for a in T for b in T])
def test_types(polyq_lib, tp, tg, bits):
    run(polyq_lib, [700, 256, 4096], T[tp], T[tg], bits)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[1], [2, 1, 255], [256], [257, 511, 512, 513], [100003], [3] * 200,
                                   [1000 + i for i in range(65)], [17] * 641, [300000, 5, 70000]])
def test_sizes(polyq_lib, sizes, bits):
    run(polyq_lib, sizes, torch.float32, torch.bfloat16, bits, copy=torch.bfloat16)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 3, 4])
def test_alignment(polyq_lib, offset, bits):
    """Tensors that start on any element."""
    run(polyq_lib, [1000, 256, 9], torch.float32, torch.float16, bits, copy=torch.float16, offset=offset)
    run(polyq_lib, [1000, 256, 9], torch.bfloat16, torch.bfloat16, bits, copy=torch.float32, offset=offset)


@pytest.mark.parametrize("bits", [32, 8])
def test_rates_of_each_tensor(polyq_lib, bits):
    run(polyq_lib, [500, 600, 700], torch.float32, torch.float32, bits, decay=[0.0, 0.1, 0.5], rate=[1.0, 0.0, 2.0])
    run(polyq_lib, [500, 600], torch.float32, torch.float32, bits, scale=torch.tensor([0.25], device="cuda"), t=1)


def test_mixed_types_in_one_plan(polyq_lib):
    """Types may differ from tensor to tensor; a tensor's copy may be missing."""
    sizes = [300, 400, 500, 600]
    a, ga, ca = tensors(sizes, torch.float32, torch.bfloat16, copy=torch.bfloat16)
    b, gb, _ = tensors(sizes, torch.float32, torch.bfloat16)
    b[1], gb[1] = b[1].bfloat16(), gb[1].float()
    a[1], ga[1] = b[1].clone(), gb[1].clone()
    ca[0] = ca[1] = None
    s, _ = random_state(polyq_lib, sizes, 32)
    polyq_lib.AdamW(a, ga, s, copies=ca).step(LR, 3)
    for i, n in enumerate(sizes):  # each alone
        s1, _ = random_state(polyq_lib, sizes, 32)
        one = polyq_lib.AdamState([n])
        one.m[:n], one.v[:n] = (x[s1.offsets[i]:s1.offsets[i] + n] for x in (s1.m, s1.v))
        polyq_lib.AdamW([b[i]], [gb[i]], one).step(LR, 3)
        assert torch.equal(a[i], b[i]) and torch.equal(one.m[:n], s.m[s.offsets[i]:s.offsets[i] + n])
        if ca[i] is not None:
            assert torch.equal(ca[i], a[i].bfloat16())


@pytest.mark.parametrize("bits", [32, 8])
def test_grad_scale_that_is_not_finite_skips_the_step(polyq_lib, bits):
    sizes = [700, 3]
    p, g, _ = tensors(sizes, torch.float32, torch.float32)
    s, _ = random_state(polyq_lib, sizes, bits)
    old = [t.clone() for t in (*p, s.m, s.v)]
    plan = polyq_lib.AdamW(p, g, s)
    for v in (float("inf"), float("-inf"), float("nan")):
        plan.step(LR, 1, grad_scale=torch.tensor([v], device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(old, (*p, s.m, s.v)))


def test_not_finite_gradients(polyq_lib):
    """32 bits: they stay with their element; 8 bits: with their block."""
    for bits in (32, 8):
        p, g, _ = tensors([600], torch.float32, torch.float32)
        g[0][300] = float("inf")
        s, _ = random_state(polyq_lib, [600], bits)
        polyq_lib.AdamW(p, g, s).step(LR, 1)
        bad = ~torch.isfinite(p[0])
        assert bad.sum() <= 1 and not bad[:300].any()
        if bits == 8:
            m, r = s.values()
            assert torch.isnan(m[256:512]).all() and torch.isnan(r[256:512]).all()
            assert torch.isfinite(m[:256]).all() and torch.isfinite(m[512:]).all()
            assert int(s.m_scales[1]) == 255 and not s.m[256:512].any()


def test_extreme_magnitudes_in_8_bits(polyq_lib):
    """Moments from subnormal to nearly the largest: scales at both ends, and blocks of zeros."""
    sizes = [256 * 5]
    p, g, _ = tensors(sizes, torch.float32, torch.float32)
    mags = [0.0, 1e-45, 1e-39, 1e-3, 1e18]
    for i, v in enumerate(mags):
        g[0][256 * i:256 * i + 256] = v * torch.linspace(0.5, 1, 256, device="cuda")
    s = polyq_lib.AdamState(sizes, 8)
    polyq_lib.AdamW(p, g, s).step(0.0, 1, betas=(0.0, 0.0))
    m, r = (x.float().view(5, 256) for x in s.values())
    want = g[0].view(5, 256)
    assert (m[0] == 0).all() and (r[0] == 0).all()
    assert ((m[3:] - want[3:]).abs() <= want[3:] / 8).all() and ((r[3:] - want[3:]).abs() <= want[3:] / 16).all()
    # units at the lowest scale: 2^-130 for m; the squares of 1e-39 are 0 in fp32
    assert ((m[1:3] - want[1:3]).abs() <= want[1:3] / 8 + 2.0 ** -130).all() and (r[1:3] == 0).all()


def test_rounding_is_unbiased(polyq_lib):
    """The mean over many seeds of what an 8-bit moment becomes is the moment: 512 seeds' fractions
    have a standard error of at most 0.5 / sqrt(512) of a step; five of them, and the mean over a
    block's elements much nearer."""
    n, seeds = 2048, 512
    g = [torch.linspace(1.0, 1.99, n, device="cuda")]
    p, total, roots = [torch.zeros(n, device="cuda")], 0, 0
    for k in range(seeds):
        s = polyq_lib.AdamState([n], 8)
        polyq_lib.AdamW(p, g, s).step(0.0, 1, betas=(0.0, 0.0), seed=k)
        m, r = s.values()
        total, roots = total + m.double(), roots + r.double()
    for mean, place in ((total / seeds, 1 / 8), (roots / seeds, 1 / 16)):
        off = ((mean - g[0].double()) / place).cpu().numpy()
        assert np.abs(off).max() <= 5 * 0.5 / np.sqrt(seeds)
        assert abs(off.mean()) <= 5 * 0.5 / np.sqrt(seeds * len(off)) + 1e-4


def test_captured_steps_take_rates_from_the_device(polyq_lib):
    """A graph's replays count the step and read the rate on the device, as separate calls do."""
    sizes = [3000, 41]
    for bits in (32, 8):
        a, ga, _ = tensors(sizes, torch.float32, torch.float32)
        b, gb, _ = tensors(sizes, torch.float32, torch.float32)
        sa, sb = polyq_lib.AdamState(sizes, bits), polyq_lib.AdamState(sizes, bits)
        pa, pb = polyq_lib.AdamW(a, ga, sa), polyq_lib.AdamW(b, gb, sb)
        lr = torch.tensor([0.0], device="cuda")
        step = torch.tensor([0], dtype=torch.int64, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step.add_(1)
            pa.step(lr, step, seed=9)
        for t in (1, 2, 3):
            lr.fill_(LR * t)
            graph.replay()
            pb.step(LR * t, t, seed=9 + t)
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            # the bias corrections are computed apart, both within a few units
            assert ((x - y).abs() <= 3 * (16 * F.U * LR * 3 * 4 + 2 * F.U * y.abs())).all()
        x, y = (sa.m, sb.m) if bits == 32 else (sa.values()[0], sb.values()[0])
        assert torch.equal(x, y)


def test_other_stream_and_repeat(polyq_lib):
    sizes = [5000, 6000]
    out = []
    for k in range(2):
        p, g, _ = tensors(sizes, torch.float32, torch.bfloat16)
        s = polyq_lib.AdamState(sizes, 8)
        plan = polyq_lib.AdamW(p, g, s)
        st = torch.cuda.Stream() if k else None
        if k:
            st.wait_stream(torch.cuda.current_stream())
        for t in (1, 2):
            plan.step(LR, t, seed=t, stream=st)
        if k:
            torch.cuda.current_stream().wait_stream(st)
        out.append((*p, s.m, s.v))
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_state_past_a_tensor_is_zero(polyq_lib):
    """The rest of a tensor's last block holds nothing, whatever was there."""
    s, _ = random_state(polyq_lib, [300], 8)
    p, g, _ = tensors([300], torch.float32, torch.float32)
    polyq_lib.AdamW(p, g, s).step(LR, 1)
    m, r = s.values()
    assert not s.m[300:].any() and not s.v[300:].any() and not m[300:].any() and not r[300:].any()


def test_moments_are_rounded_after_each_operation(polyq_lib):
    """m = b1 m + (1-b1) g and v = b2 v + ((1-b2) g) g, each product and sum rounded by itself: the
    codes of an 8-bit state follow from this order, so that no product and sum may be one rounding."""
    n, b1, b2 = 1 << 20, 0.9, 0.95
    gen = torch.Generator("cuda").manual_seed(7)
    p, g, m, v = (torch.randn(n, generator=gen, device="cuda") * s for s in (0.02, 1e-3, 1e-3, 1e-3))
    state = polyq_lib.AdamState([n], bits=32)
    state.m.copy_(m)
    state.v.copy_(v.square())
    one_b1, one_b2 = (torch.tensor(1 - b, dtype=torch.float64).float().cuda() for b in (b1, b2))
    want_m = m * torch.tensor(b1).cuda() + one_b1 * g
    want_v = v.square() * torch.tensor(b2).cuda() + (one_b2 * g) * g
    polyq_lib.AdamW([p], [g], state).step(lr=1e-3, step=3, betas=(b1, b2))
    assert torch.equal(state.m, want_m) and torch.equal(state.v, want_v)
