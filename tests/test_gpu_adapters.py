"""GPU tests of the low-rank adapters, forward and backward, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import finetune_util as F
from tests.fp4_util import dense

pytestmark = pytest.mark.gpu
T16 = {"bf16": torch.bfloat16, "f16": torch.float16}


def within(got, ref, bound, what, rows=None):
    got = got.double()
    if rows is not None:
        got, ref, bound = got[rows], ref[rows], bound[rows]
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - ref).abs() - bound
    assert (over <= 0).all(), f"{what}: {(over > 0).sum()} off, worst {over.max():.3g} over the bound"


def make(T, K, N, R, n, dtype, seed=0, pad=0, out=None, x_scale=1.0, xpad=None):
    g = torch.Generator("cuda").manual_seed(seed)

    def rnd(*s):
        return torch.randn(*s, generator=g, device="cuda")

    x = dense(T, K, dtype, (-K) % 8 + 8 * pad if xpad is None else xpad[0], 0 if xpad is None else xpad[1])
    x.copy_(rnd(T, K) * x_scale)
    dy = dense(T, N, dtype, (-N) % 8 + 8 * pad if xpad is None else xpad[0], 0 if xpad is None else xpad[1])
    dy.copy_(rnd(T, N))
    a = torch.zeros(n, R, K + (-K) % 8 + 8 * pad, dtype=dtype, device="cuda")[:, :, :K]
    a.copy_(rnd(n, R, K) * K ** -0.5)
    b = torch.zeros(n, N, R + 8 * pad, dtype=dtype, device="cuda")[:, :, :R]
    b.copy_(rnd(n, N, R) * 0.1)
    return x, a, b, dy, rnd(T, N), rnd(T, K)


def segments(lengths, first=0):
    off = np.concatenate([[first], first + np.cumsum(lengths)]).astype(int).tolist()
    return off, torch.tensor(off, dtype=torch.int32, device="cuda")


def run(polyq, lengths, ids, T, K, N, R, n, dtype=torch.bfloat16, out=None, dxt=None, gt=torch.float32, ranks=None,
        pad=0, ypad=0, first=0, seed=0, in_place=False, train=True, x_scale=1.0, residual=True,
        xpad=None):
    out, dxt = out or dtype, dxt or dtype
    x, a, b, dy, y0, dx0 = make(T, K, N, R, n, dtype, seed, pad, x_scale=x_scale, xpad=xpad)
    off, d_off = segments(lengths, first)
    d_ids = torch.tensor(ids, dtype=torch.int32, device="cuda")
    r = np.random.default_rng(seed)
    scales = [float(2.0 * r.random()) for _ in range(n)]
    d_scales = torch.tensor(scales, device="cuda")
    scales = d_scales.tolist()
    rk = [R] * n if ranks is None else ranks
    d_ranks = None if ranks is None else torch.tensor(ranks, dtype=torch.int32, device="cuda")
    for i, k in enumerate(rk):  # what lies past a rank does not matter
        a[i, k:], b[i, :, k:] = float("nan"), float("inf")
    res, y = dense(T, N, out, ypad), dense(T, N, out, ypad)
    res.copy_(y0)
    if in_place:
        y = res.clone() if not ypad else res
    base = (res.double() if residual else torch.zeros(T, N, dtype=torch.float64, device="cuda"))
    before = y.clone()
    saved = polyq.adapters_saved(T, R)
    polyq.adapters_forward(x, a, b, d_off, d_ids, scales=d_scales, ranks=d_ranks,
                           residual=(y if in_place else res) if residual else None, y=y, saved=saved)
    dres = dense(T, K, dxt, ypad)
    dres.copy_(dx0)
    ref = F.adapters(x, a, b, off, ids, scales, rk, base, dy, dres.double(), out, dxt, gt)
    rows = slice(off[0], off[-1])
    within(y, *ref[0], "y", rows)
    for part in (slice(0, off[0]), slice(off[-1], T)):  # rows of no segment
        assert torch.equal(y[part].nan_to_num(7.0), before[part].nan_to_num(7.0))
    if not train:
        return y
    dx = dense(T, K, dxt, ypad)
    da, db = (torch.full((n, *s), float("nan"), dtype=gt, device="cuda") for s in ((R, K), (N, R)))
    polyq.adapters_backward(x, a, b, saved, dy, d_off, d_ids, scales=d_scales, ranks=d_ranks, residual=dres, dx=dx,
                            da=da, db=db)
    within(dx, *ref[1], "dx", rows)
    assert torch.isnan(dx[:off[0]]).all() and torch.isnan(dx[off[-1]:]).all()
    within(da, *ref[2], "da")
    within(db, *ref[3], "db")
    return y


@pytest.mark.parametrize("dtype", list(T16))
@pytest.mark.parametrize("out", ["x", "f32"])
@pytest.mark.parametrize("R", [8, 16, 24, 32, 40, 64, 72, 128])
def test_ranks_and_types(polyq_lib, R, out, dtype):
    t = T16[dtype]
    o = t if out == "x" else torch.float32
    run(polyq_lib, [5, 60, 100, 35], [1, 0, -1, 2], 200, 136, 200, R, 3, t, out=o, dxt=o, gt=o,
        ranks=[R, R - 3, max(1, R // 2)])


@pytest.mark.parametrize("dtype", list(T16))
@pytest.mark.parametrize("lengths,ids,n", [
    ([1], [0], 1), ([1, 1, 1, 1, 1], [4, 0, 2, 2, 1], 5), ([3, 0, 7, 0, 0, 1], [0, 1, 0, 1, 0, 1], 2),
    ([16, 17, 15, 33], [0, 1, 0, 1], 2), ([64, 65, 63, 128, 129, 1], [2, 0, 1, 0, 2, 1], 3), ([700], [0], 1),
    ([1] * 70, list(range(70)), 70), ([2, 1] * 33, [-1, 0] * 33, 1), ([513, 300], [0, 0], 2),
    ([40, 41, 42], [7, -5, 100], 3), ([0, 0], [0, 1], 2)])
def test_segments(polyq_lib, lengths, ids, n, dtype):
    T = max(1, sum(lengths))
    run(polyq_lib, lengths, ids, T, 320, 264, 16, n, T16[dtype])
    run(polyq_lib, lengths, ids, T + 9, 200, 520, 64, n, T16[dtype], first=4, out=torch.float32)


@pytest.mark.parametrize("K,N", [(1, 1), (7, 9), (8, 8), (63, 65), (129, 1000), (1001, 255), (4096, 257), (72, 4099),
                                 (2056, 2048)])
@pytest.mark.parametrize("lengths", [[9, 3], [150, 70]])
def test_sizes(polyq_lib, K, N, lengths):
    run(polyq_lib, lengths, [1, 0], sum(lengths), K, N, 16, 2)
    run(polyq_lib, lengths, [1, 0], sum(lengths), K, N, 32, 2, torch.float16, ranks=[32, 5])


@pytest.mark.parametrize("R", [16, 64, 128])
def test_long_sequences(polyq_lib, R):
    run(polyq_lib, [1000, 1500, 37], [0, 1, 0], 2537, 1024, 1504, R, 2)
    run(polyq_lib, [2100], [0], 2100, 520, 640, R, 1, torch.float16, gt=torch.float16)


@pytest.mark.parametrize("pad,ypad", [(1, 0), (0, 1), (2, 8), (0, 5)])
def test_strides(polyq_lib, pad, ypad):
    for lengths in ([3, 4], [70, 90]):
        run(polyq_lib, lengths, [0, 1], sum(lengths), 200, 304, 24, 2, pad=pad, ypad=ypad)
        run(polyq_lib, lengths, [0, 1], sum(lengths), 200, 304, 24, 2, pad=pad, ypad=ypad, out=torch.float32)


@pytest.mark.parametrize("dtype", list(T16))
@pytest.mark.parametrize("R", [8, 32, 64, 128])
@pytest.mark.parametrize("K,N,xpad", [(1000, 321, (0, 0)), (133, 1001, (0, 0)), (64, 128, (1, 0)), (64, 128, (0, 1)),
                                      (200, 135, (3, 5))])
def test_rows_that_start_anywhere(polyq_lib, K, N, xpad, R, dtype):
    """x and dy of odd widths without gaps, and of buffers that start on any element."""
    for lengths, ids in (([9, 1, 14], [1, 0, -1]), ([150, 70, 33], [0, 1, 0])):
        run(polyq_lib, lengths, ids, sum(lengths) + 2, K, N, R, 2, T16[dtype], xpad=xpad, ranks=[R, max(1, R - 3)])


@pytest.mark.parametrize("lengths", [[3, 4, 2], [70, 90, 10]])
def test_in_place_and_without_residual(polyq_lib, lengths):
    ids, T = [0, -1, 1], sum(lengths)
    a = run(polyq_lib, lengths, ids, T, 128, 256, 16, 2, train=False)
    b = run(polyq_lib, lengths, ids, T, 128, 256, 16, 2, train=False, in_place=True)
    assert torch.equal(a, b)
    c = run(polyq_lib, lengths, ids, T, 128, 256, 16, 2, train=False, residual=False)
    assert (c[lengths[0]:lengths[0] + lengths[1]] == 0).all()


def test_fp16_keeps_magnitudes_out_of_its_range(polyq_lib):
    """v far above and below fp16's numbers: in fp32 between the products."""
    for scale in (60.0, 2.0 ** -12):
        g = torch.Generator("cuda").manual_seed(3)
        x = (torch.randn(100, 512, generator=g, device="cuda") * scale).half()
        a = (torch.randn(1, 16, 512, generator=g, device="cuda") * (100.0 if scale > 1 else 2.0 ** -12)).half()
        b = (torch.randn(1, 128, 16, generator=g, device="cuda") * 2.0 ** -9).half()
        dy = torch.randn(100, 128, generator=g, device="cuda").half()
        off, d_off = segments([100])
        ids = torch.zeros(1, dtype=torch.int32, device="cuda")
        saved = polyq_lib.adapters_saved(100, 16)
        y = polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved, dtype=torch.float32)
        assert saved.abs().max() > 70000 if scale > 1 else saved.abs().max() < 2.0 ** -15
        z = torch.zeros(100, 128, dtype=torch.float64, device="cuda")
        zx = torch.zeros(100, 512, dtype=torch.float64, device="cuda")
        ref = F.adapters(x, a, b, off, [0], [1.0], [16], z, dy, zx, torch.float32, torch.float32, torch.float32)
        got = polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids, dx=zx.float(),
                                          da=torch.empty(a.shape, device="cuda"), db=torch.empty(b.shape, device="cuda"))
        for v, r, what in zip((y, *got), ref, ("y", "dx", "da", "db")):
            within(v, *r, what)


@pytest.mark.parametrize("dtype", list(T16))
@pytest.mark.parametrize("lengths", [[4, 5, 6], [80, 90, 70]])
def test_not_finite_rows_stay_apart(polyq_lib, lengths, dtype):
    """A row that is not finite reaches its own outputs and its adapter's gradients only."""
    t = T16[dtype]
    T = sum(lengths)
    x, a, b, dy, y0, _ = make(T, 128, 192, 16, 3, t)
    _, d_off = segments(lengths)
    ids = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")

    def step():
        saved = polyq_lib.adapters_saved(T, 16)
        y = polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved)
        return (y, *polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids))

    good = step()
    row = lengths[0] + 1  # of adapter 1
    x[row, 3], dy[row, 5] = float("nan"), float("inf")
    bad = step()
    keep = torch.arange(T, device="cuda") != row
    for i in (0, 1):
        assert torch.equal(good[i][keep], bad[i][keep]) and not torch.isfinite(bad[i][row]).all()
    for i in (2, 3):
        assert torch.equal(good[i][[0, 2]], bad[i][[0, 2]]) and not torch.isfinite(bad[i][1]).all()
    # ranks: what is past one stays zero
    ranks = torch.tensor([16, 3, 16], dtype=torch.int32, device="cuda")
    saved = polyq_lib.adapters_saved(T, 16)
    polyq_lib.adapters_forward(x, a, b, d_off, ids, ranks=ranks, saved=saved)
    _, da, db = polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids, ranks=ranks)
    assert (da[1, 3:] == 0).all() and (db[1, :, 3:] == 0).all()


@pytest.mark.parametrize("dtype", list(T16))
@pytest.mark.parametrize("lengths", [[4, 5, 6], [80, 90, 70]])
def test_a_rank_that_is_not_finite_stays_apart(polyq_lib, lengths, dtype):
    """An infinity in one rank's row of a, or column of b, leaves the other ranks' gradients as
    zeros there would."""
    t = T16[dtype]
    T = sum(lengths)
    x, a, b, dy, _, _ = make(T, 128, 192, 16, 3, t)
    _, d_off = segments(lengths)
    ids = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")

    def step():
        saved = polyq_lib.adapters_saved(T, 16)
        polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved)
        return polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids)[1:]

    a[1, 3], b[1, :, 5] = 0, 0
    good = step()
    a[1, 3, 7], b[1, 11, 5] = float("inf"), float("-inf")
    da, db = step()
    others = [j for j in range(16) if j not in (3, 5)]
    assert not torch.isfinite(da[1, 5]).any() and not torch.isfinite(db[1, :, 3]).any()
    assert torch.equal(da[:, others], good[0][:, others]) and torch.equal(db[:, :, others], good[1][:, :, others])
    assert torch.equal(da[[0, 2]], good[0][[0, 2]]) and torch.equal(db[[0, 2]], good[1][[0, 2]])


def test_offsets_outside_the_rows_are_held(polyq_lib):
    """Segments past the tensors' end or before their start keep inside; a falling pair is empty."""
    x, a, b, dy, _, _ = make(50, 128, 192, 16, 2, torch.bfloat16)
    ids = torch.tensor([0, 1, 0], dtype=torch.int32, device="cuda")
    off = torch.tensor([-7, 20, 60, 1 << 30], dtype=torch.int32, device="cuda")
    held = torch.tensor([0, 20, 50, 50], dtype=torch.int32, device="cuda")
    out = []
    for o in (off, held):
        saved = polyq_lib.adapters_saved(50, 16)
        y = polyq_lib.adapters_forward(x, a, b, o, ids, saved=saved)
        out.append((y, *polyq_lib.adapters_backward(x, a, b, saved, dy, o, ids)))
    assert all(torch.equal(p, q) for p, q in zip(*out))
    fall = torch.tensor([30, 10, 10, 50], dtype=torch.int32, device="cuda")
    y = polyq_lib.adapters_forward(x, a, b, fall, ids, y=torch.full((50, 192), 3.0, dtype=x.dtype, device="cuda"))
    assert (y[:10] == 3).all() and (y[10:] != 3).any()


def test_ranks_outside_their_range_are_held(polyq_lib):
    x, a, b, dy, _, _ = make(20, 128, 192, 16, 2, torch.bfloat16)
    _, d_off = segments([10, 10])
    ids = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    y = [polyq_lib.adapters_forward(x, a, b, d_off, ids, ranks=torch.tensor(r, dtype=torch.int32, device="cuda"))
         for r in ([99, -4], [16, 0])]
    assert torch.equal(*y) and (y[0][10:] == 0).all()


def test_chosen_gradients(polyq_lib):
    x, a, b, dy, _, _ = make(150, 136, 200, 24, 2, torch.bfloat16)
    _, d_off = segments([50, 100])
    ids = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    saved = polyq_lib.adapters_saved(150, 24)
    polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved)
    every = polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids)
    dx, da, db = polyq_lib.adapters_backward(x, a, b, None, dy, d_off, ids, need_weights=False)
    assert da is None and db is None and torch.equal(dx, every[0])
    dx, da, db = polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids, need_dx=False)
    assert dx is None and torch.equal(da, every[1]) and torch.equal(db, every[2])
    fresh = polyq_lib.adapters_forward(x, a, b, d_off, ids)
    assert torch.equal(fresh, polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved))


@pytest.mark.parametrize("lengths", [[2, 1, 1], [90, 200, 77]])
def test_replayed_graph_with_other_segments(polyq_lib, lengths):
    """Offsets, ids, ranks and scales are read when a captured call runs; results repeat bit for bit."""
    T = sum(lengths)
    x, a, b, dy, y0, dx0 = make(T, 264, 328, 32, 3, torch.bfloat16)
    off = segments(lengths)[1]
    ids = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    scales, ranks = torch.ones(3, device="cuda"), torch.full((3,), 32, dtype=torch.int32, device="cuda")
    res = y0.bfloat16()

    def step(**kw):
        saved = kw.pop("saved")
        y = polyq_lib.adapters_forward(x, a, b, off, ids, scales=scales, ranks=ranks, residual=res, saved=saved, **kw)
        return (y, *polyq_lib.adapters_backward(x, a, b, saved, dy, off, ids, scales=scales, ranks=ranks,
                                                residual=dx0.bfloat16(), **kw))

    saved = polyq_lib.adapters_saved(T, 32)
    first = step(saved=saved)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        again = step(saved=saved)
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    off.copy_(torch.tensor([0, 1, T - 1, T]))
    ids.copy_(torch.tensor([2, 0, -1]))
    scales.fill_(0.5)
    ranks.copy_(torch.tensor([5, 32, 17]))
    g.replay()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    apart = step(saved=polyq_lib.adapters_saved(T, 32), stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(apart, again)) and not torch.equal(first[0], again[0])


def test_gradients_against_differences(polyq_lib):
    """Central differences of sum(y dy) in a; the output is linear in it, so the only errors are the
    outputs' (fp32, each within its bound) and a's step, which bf16 holds."""
    lengths, T = [6, 10], 16
    x, a, b, dy, _, _ = make(T, 64, 48, 8, 2, torch.bfloat16)
    off, d_off = segments(lengths)
    ids = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    a = (a * 16).round() / 16
    saved = polyq_lib.adapters_saved(T, 8)
    polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved)
    _, da, db = polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids, da=torch.empty(a.shape, device="cuda"),
                                            db=torch.empty(b.shape, device="cuda"))
    zero = torch.zeros(T, 48, dtype=torch.float64, device="cuda")

    def loss(a_, b_):
        y = polyq_lib.adapters_forward(x, a_, b_, d_off, ids, dtype=torch.float32)
        bound = F.adapters(x, a_, b_, off, [1, 0], [1.0, 1.0], [8, 8], zero, out=torch.float32)[0][1]
        return float((y.double() * dy.double()).sum()), float((bound * dy.double().abs()).sum())

    b = (b * 16).round() / 16
    saved = polyq_lib.adapters_saved(T, 8)
    polyq_lib.adapters_forward(x, a, b, d_off, ids, saved=saved)
    _, da, db = polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, ids, da=torch.empty(a.shape, device="cuda"),
                                            db=torch.empty(b.shape, device="cuda"))
    for which, t, g in ((0, a, da), (1, b, db)):
        for i in range(0, t.numel(), 97):
            vals = []
            for h in (0.25, -0.25):
                u = t.clone()
                u.view(-1)[i] += h
                vals.append(loss(*((u, b) if which == 0 else (a, u))))
            num = (vals[0][0] - vals[1][0]) / 0.5
            own = 2.0 ** -16 * float(g.abs().max())
            assert abs(num - float(g.view(-1)[i])) <= (vals[0][1] + vals[1][1]) / 0.5 + own, (which, i)
