"""GPU tests of AdamW over many steps and of what its plans hold."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_default_rounding_follows_the_moments_over_time(polyq_lib):
    """300 steps of a zero gradient from a state of equal elements: the mean of m is beta1^t of what it
    was, that of the root beta2^(t/2).

    A rounding by chance is off by 0 on average (by 2^-16 of a code's step at most, of which 300 are
    5.7e-4) and has a variance of a quarter of that step squared at most, which is 2^-3 of m's
    magnitudes and 2^-4 of the root's: over the steps a relative variance of (1 + 2^-8)^300 - 1 for m
    and (1 + 2^-10)^300 - 1 for the root, of each of 65536 elements."""
    n, steps, b1, b2 = 1 << 16, 300, 0.9, 0.999
    g = [torch.full((n,), 1e-3, device="cuda")]
    p, s = [torch.zeros(n, device="cuda")], polyq_lib.AdamState([n], 8)
    plan = polyq_lib.AdamW(p, g, s)
    plan.step(1e-3, 1, betas=(b1, b2))
    before = [float(v.double().mean()) for v in s.values()]
    g[0].zero_()
    for t in range(2, steps + 2):
        plan.step(1e-3, t, betas=(b1, b2))
    after = [float(v.double().mean()) for v in s.values()]
    for what, old, new, keep, place in (("m", before[0], after[0], b1 ** steps, 1 / 8),
                                        ("root", before[1], after[1], b2 ** (steps / 2), 1 / 16)):
        sigma = np.sqrt(((1 + place ** 2 / 4) ** steps - 1) / n)
        assert abs(new / (old * keep) - 1) <= 6 * sigma + 6e-4, (what, old, new, keep)


def test_default_rounding_is_that_of_a_step_on_the_device(polyq_lib):
    """The number of the step gives the same codes from the host and from the device."""
    n = 5000
    gen = torch.Generator("cuda").manual_seed(3)
    out = []
    for on_device in (False, True):
        p, s = [torch.zeros(n, device="cuda")], polyq_lib.AdamState([n], 8)
        g = [torch.randn(n, generator=gen.manual_seed(3), device="cuda")]
        plan = polyq_lib.AdamW(p, g, s)
        for t in (1, 2, 3):
            plan.step(1e-3, torch.tensor([t], device="cuda") if on_device else t)
        out.append([s.m, s.v, s.m_scales, s.v_scales])
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("bits", [32, 8])
def test_smallest_eps(polyq_lib, bits):
    """Where m and v are 0 a parameter only decays, with the smallest eps too."""
    p, g = [torch.full((700,), 2.0, device="cuda")], [torch.zeros(700, device="cuda")]
    polyq_lib.AdamW(p, g, polyq_lib.AdamState([700], bits), weight_decay=0.5).step(0.25, 1, eps=2.0 ** -126)
    assert torch.equal(p[0], torch.full_like(p[0], 2.0 * (1 - 0.25 * 0.5)))


def test_replaced_gradients_are_refused(polyq_lib):
    """A plan over parameters' own .grad does not go on with gradients that have been replaced."""
    ps = [torch.ones(300, device="cuda", requires_grad=True) for _ in range(3)]

    def backward():
        sum((k + 1) * p.sum() for k, p in enumerate(ps)).backward()

    def plan():
        return polyq_lib.AdamW(ps, [p.grad for p in ps], state)

    state = polyq_lib.AdamState([300] * 3)
    opt = torch.optim.SGD(ps)
    backward()
    adam = plan()
    adam.step(1e-3, 1)
    opt.zero_grad(set_to_none=False)
    ps[1].grad = ps[1].grad.view(300)  # (the same memory)
    backward()
    adam.step(1e-3, 2)
    before = [p.detach().clone() for p in ps] + [state.m.clone()]
    opt.zero_grad()  # to None
    for make in (lambda: None, backward):
        make()
        with pytest.raises(ValueError, match="no longer"):
            adam.step(1e-3, 3)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, [p.detach() for p in ps] + [state.m]))
    plan().step(1e-3, 3)
    assert all((p.detach() < b).all() for p, b in zip(ps, before))
    # gradients beside .grad are the caller's own
    mine = [torch.ones(300, device="cuda") for _ in ps]
    adam = polyq_lib.AdamW(ps, mine, state)
    opt.zero_grad()
    adam.step(1e-3, 4)


def test_a_plan_keeps_its_memory(polyq_lib):
    """Tensors that are given other memory leave the plan with what it has laid out."""
    n = 1 << 20
    p, g, c = (torch.ones(n, device="cuda", dtype=t) for t in (torch.float32, torch.float32, torch.bfloat16))
    old = [t.data_ptr() for t in (p, g, c)]
    adam = polyq_lib.AdamW([p], [g], polyq_lib.AdamState([n]), copies=[c])
    for t in (p, g, c):
        t.data = torch.full_like(t, 5)
    others = [torch.full((n,), 7, device="cuda", dtype=t) for _ in range(4) for t in (torch.float32, torch.bfloat16)]
    assert not {t.data_ptr() for t in others} & set(old)
    adam.step(1e-3, 1)
    assert all((t == 7).all() for t in others) and all((t == 5).all() for t in (p, g, c))


def test_shared_memory_is_refused(polyq_lib):
    """Two updates of one element at the same time would give either's result."""
    buf, g = torch.ones(1000, device="cuda"), [torch.ones(300, device="cuda") for _ in range(2)]
    state = polyq_lib.AdamState([300] * 2)
    for ps, cs in (([buf[:300]] * 2, None), ([buf[:300], buf[299:599]], None), ([buf[600:900], buf[:300]], [buf[500:800], None]),
                   ([buf[:300], buf[300:600]], [buf[600:900], buf[600:900]])):
        with pytest.raises(ValueError, match="share memory"):
            polyq_lib.AdamW(ps, g, state, copies=cs)
    polyq_lib.AdamW([buf[300:600], buf[:300]], g, state, copies=[None, buf[600:900]]).step(1e-3, 1)
    assert (buf[:900] < 1).all() and (buf[900:] == 1).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_gradient_that_is_not_finite_reaches_its_own_parameter(polyq_lib, bits, value):
    p, g = [torch.ones(600, device="cuda")], [torch.full((600,), 1e-2, device="cuda")]
    g[0][300] = value
    polyq_lib.AdamW(p, g, polyq_lib.AdamState([600], bits)).step(1e-3, 1)
    assert (~torch.isfinite(p[0])).nonzero().flatten().tolist() == [300]
