"""GPU tests of layer norm and RMS norm, forward and backward, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import finetune_util as F
from tests.fp4_util import check, dense, f64, put

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def inputs(rows, K, tx, ty, seed, pad=(0, 0), offset=0, shift=0.3):
    r = np.random.default_rng(seed)
    m = np.exp(r.standard_normal(K)) * np.where(r.random(K) < 0.02, 20, 1)
    x = put(m * r.standard_normal((rows, K)) + shift, tx, pad[0], offset)
    dy = put(r.standard_normal((rows, K)), ty, pad[1], offset)
    res = put(r.standard_normal((rows, K)), tx, pad[0], offset)
    return x, dy, res, 1 + 0.2 * r.standard_normal(K), 0.5 * r.standard_normal(K)


def run(polyq, rows, K, tx, ty, center=True, wt=torch.float32, pad=(0, 0), offset=0, bias=True,
        residual=True, eps=1e-5, seed=0):
    x, dy, res, w, b = inputs(rows, K, tx, ty, seed, pad, offset)
    tw, tb = (torch.from_numpy(v).to("cuda", wt) for v in (w, b))
    stats = polyq.layernorm_stats(rows)
    y = dense(rows, K, ty, pad[1], offset)
    polyq.layernorm_forward(x, tw, tb if bias else None, eps=eps, center=center, y=y, stats=stats)
    X, W, B = f64(x), f64(tw), f64(tb) * bias
    ref, hat, mean, rstd = F.norm(X, W, B, eps, center)
    check(f64(y), ref, F.norm_bound(X, W, B, ref, hat, rstd, center, ty), "y")
    st = f64(stats)
    check(st[:, :1], mean, 30 * F.U * np.abs(X).mean(1, keepdims=True), "mean")
    check(st[:, 1:], rstd, rstd * (20 * F.U + (30 * F.U * np.abs(X).mean(1, keepdims=True) * rstd) ** 2), "rstd")
    dx = dense(rows, K, tx, pad[0], offset)
    got = polyq.layernorm_backward(x, tw, stats, dy, center=center, dx=dx,
                                   residual=res if residual else None)
    R = f64(res) * residual
    refs = F.norm_backward(X, W, f64(dy), R, eps, center)
    bounds = F.norm_backward_bounds(X, W, f64(dy), R, eps, center, tx, wt)
    for g, r_, e, what in zip(got, refs, bounds, ("dx", "dw", "db")):
        check(f64(g), r_, e, what)
    return x, y, dx


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("tx,ty", [(a, b) for a in T for b in T])
def test_types(polyq_lib, tx, ty, center):
    run(polyq_lib, 37, 520, T[tx], T[ty], center)


@pytest.mark.parametrize("rows,K", [(1, 1), (1, 5120), (5, 7), (3, 8), (2, 255), (2, 256), (2, 257), (700, 64),
                                    (1000, 31), (5000, 33), (613, 1000), (40, 5003), (9, 6144), (9, 6145),
                                    (4, 8192), (4, 8193), (3, 16384), (2, 20001), (2, 24576), (1, 24575)])
@pytest.mark.parametrize("center", [True, False])
def test_sizes(polyq_lib, rows, K, center):
    run(polyq_lib, rows, K, torch.bfloat16, torch.bfloat16, center, seed=rows + K)
    if rows * K < 100000:
        run(polyq_lib, rows, K, torch.float32, torch.float32, center, seed=rows + K)


def test_many_rows(polyq_lib):
    run(polyq_lib, 20001, 72, torch.float16, torch.float16)
    run(polyq_lib, 3001, 640, torch.bfloat16, torch.float32, False)


@pytest.mark.parametrize("pad,offset", [((8, 16), 0), ((8, 3), 0), ((1, 0), 0), ((0, 0), 1), ((3, 5), 7)])
def test_strides_and_alignment(polyq_lib, pad, offset):
    """Rows of wider buffers, and buffers that start anywhere; what lies between rows stays."""
    for K in (1001, 1000):
        x, y, dx = run(polyq_lib, 11, K, torch.bfloat16, torch.bfloat16, pad=pad, offset=offset)
        for t, p in ((y, pad[1]), (dx, pad[0])):
            if p:
                wide = t.as_strided((10, p), (K + p, 1), t.storage_offset() + K)
                assert torch.isnan(wide).all()


@pytest.mark.parametrize("wt", list(T))
def test_weight_types(polyq_lib, wt):
    run(polyq_lib, 50, 300, torch.bfloat16, torch.bfloat16, wt=T[wt])


def test_without_weight_or_bias(polyq_lib):
    run(polyq_lib, 20, 300, torch.float32, torch.bfloat16, bias=False, residual=False)
    x, dy, res, w, b = inputs(20, 300, torch.float32, torch.float32, 1)
    stats = polyq_lib.layernorm_stats(20)
    y = polyq_lib.layernorm_forward(x, stats=stats)
    one = torch.ones(300, device="cuda")
    assert torch.equal(y, polyq_lib.layernorm_forward(x, one, one * 0))
    a = polyq_lib.layernorm_backward(x, None, stats, dy)
    b = polyq_lib.layernorm_backward(x, one, stats, dy)
    assert all(torch.equal(u, v) for u, v in zip(a, b)) and a[1].dtype == torch.float32


def test_chosen_gradients(polyq_lib):
    """Each gradient alone is what it is with the others."""
    x, dy, res, w, b = inputs(130, 264, torch.bfloat16, torch.bfloat16, 2)
    tw, stats = torch.from_numpy(w).to("cuda", torch.bfloat16), polyq_lib.layernorm_stats(130)
    polyq_lib.layernorm_forward(x, tw, stats=stats)
    every = polyq_lib.layernorm_backward(x, tw, stats, dy)
    for i in range(3):
        need = [i == j for j in range(3)]
        got = polyq_lib.layernorm_backward(x, tw, stats, dy, need_dx=need[0], need_weight=need[1], need_bias=need[2])
        assert [g is not None for g in got] == need and torch.equal(got[i], every[i])
    wide = polyq_lib.layernorm_backward(x, tw, stats, dy, dweight=torch.empty(264, device="cuda"))[1]
    assert torch.equal(wide.bfloat16(), every[1])


@pytest.mark.parametrize("K", [1000, 1001, 9000])
def test_in_place(polyq_lib, K):
    """y in x's place; dx in dy's, and in the residual's."""
    x, dy, res, w, b = inputs(33, K, torch.bfloat16, torch.bfloat16, 3)
    tw, stats = torch.from_numpy(w).float().cuda(), polyq_lib.layernorm_stats(33)
    y = polyq_lib.layernorm_forward(x, tw, stats=stats)
    dx = polyq_lib.layernorm_backward(x, tw, stats, dy, residual=res)[0]
    a = dy.clone()
    assert torch.equal(polyq_lib.layernorm_backward(x, tw, stats, a, dx=a, residual=res)[0], dx)
    a = res.clone()
    assert torch.equal(polyq_lib.layernorm_backward(x, tw, stats, dy, dx=a, residual=a)[0], dx)
    a = x.clone()
    assert torch.equal(polyq_lib.layernorm_forward(a, tw, y=a), y)


def test_mean_far_from_zero(polyq_lib):
    """The mean is taken out before squares are summed: a spread of 1 around 4096."""
    r = np.random.default_rng(4)
    x = torch.from_numpy(4096 + r.standard_normal((5, 3000))).float().cuda()
    y = polyq_lib.layernorm_forward(x)
    X = f64(x)
    ref, hat, mean, rstd = F.norm(X, 1.0, 0.0, 1e-5, True)
    check(f64(y), ref, F.norm_bound(X, 1.0, 0.0, ref, hat, rstd, True, torch.float32), "y")
    flat = polyq_lib.layernorm_forward(torch.full((2, 999), 7.0, device="cuda"))
    assert (flat.abs() <= 30 * F.U * 7 / np.sqrt(1e-5)).all()


def test_not_finite_rows_stay_apart(polyq_lib):
    x, dy, res, w, b = inputs(6, 800, torch.float32, torch.float32, 5)
    good = polyq_lib.layernorm_forward(x, center=False)
    x[1, 5], x[3, 7] = float("nan"), float("inf")
    for center in (True, False):
        y = polyq_lib.layernorm_forward(x, center=center)
        assert torch.isnan(y[1]).all()
        assert torch.isnan(y[3]).all() if center else torch.isnan(y[3, 7]) and (y[3, :7] == 0).all()
    assert torch.equal(y[[0, 2, 4, 5]], good[[0, 2, 4, 5]])


def test_runs_repeat_and_graphs_replay(polyq_lib):
    """The same bits again, on another stream, and in a replayed graph with new inputs."""
    x, dy, res, w, b = inputs(900, 1504, torch.bfloat16, torch.bfloat16, 6)
    tw, ws, stats = torch.from_numpy(w).float().cuda(), polyq_lib.layernorm_workspace(900, 1504), polyq_lib.layernorm_stats(900)

    def step(**kw):
        y = polyq_lib.layernorm_forward(x, tw, stats=stats, **kw)
        return (y, *polyq_lib.layernorm_backward(x, tw, stats, y, residual=res, workspace=ws, **kw))

    a = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b_ = step(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(u, v) for u, v in zip(a, b_))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c = step()
    x.mul_(0.5)
    g.replay()
    torch.cuda.synchronize()
    d = step()
    assert all(torch.equal(u, v) for u, v in zip(c, d)) and not torch.equal(a[3], d[3])


def test_gradients_against_differences(polyq_lib):
    """Central differences of sum(y dy), in fp32 with a step whose rounding is known."""
    r = np.random.default_rng(7)
    x, w, b, dy = (torch.from_numpy(v).float().cuda() for v in
                   (r.standard_normal((4, 24)), r.standard_normal(24), r.standard_normal(24),
                    r.standard_normal((4, 24))))
    stats = polyq_lib.layernorm_stats(4)
    polyq_lib.layernorm_forward(x, w, b, stats=stats)
    dx, dw, db = polyq_lib.layernorm_backward(x, w, stats, dy)

    def loss(**kw):
        a = dict(x=x, w=w, b=b, **{})
        a.update(kw)
        return float((polyq_lib.layernorm_forward(a["x"], a["w"], a["b"]).double() * dy.double()).sum())

    # the loss sums 96 terms of under 20, each off by 100 U at most: 0.012 over a step of 2 * 2^-6
    # is under 4e-1 * 2^-6; the third derivative (under 50 here) adds 50 h^2 / 6
    h = 2.0 ** -6
    bound = 96 * 20 * 100 * F.U / h + 50 * h * h / 6
    for name, t, g in (("x", x, dx), ("w", w, dw), ("b", b, db)):
        for i in range(0, t.numel(), 5):
            up, down = t.clone(), t.clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            num = (loss(**{name: up}) - loss(**{name: down})) / (2 * h)
            assert abs(num - float(g.view(-1)[i])) <= bound, (name, i)
