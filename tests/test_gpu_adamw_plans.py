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
