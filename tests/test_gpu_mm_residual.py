"""GPU tests of residuals: of tiles that several pairs share along the
contraction, and of a chain of short calls each of which adds to what the launch
before it wrote."""
import pytest

from tests.fp4_util import U32, dense, half_step, tiny

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

MX, NV = 0, 1


def _q(polyq, g, rows, K, fmt, scale=0.1):
    x = torch.randn(rows, K, generator=g, device="cuda") * scale
    return polyq.fp4_quantize(x, fmt, 1.0 if fmt == MX else 2.0 ** -8)


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N,K", [(2304, 2560, 13824), (2300, 2500, 7000), (7424, 1024, 40000)])
def test_shared_tiles(polyq_lib, fmt, M, N, K):
    """Rows of every alignment, each type, also in place."""
    g = torch.Generator("cuda").manual_seed(M + N)
    x, w = _q(polyq_lib, g, M, K, fmt), _q(polyq_lib, g, N, K, fmt)
    xv, wv = (polyq_lib.fp4_dequantize(t).double() for t in (x, w))
    prod, S = xv @ wv.T, xv.abs() @ wv.abs().T
    del xv, wv
    for t, pad, offset in ((torch.bfloat16, 0, 0), (torch.bfloat16, 3, 1), (torch.float16, 4, 4),
                           (torch.float32, 0, 0), (torch.float32, 1, 1)):
        res = dense(M, N, t, pad, offset)
        res.copy_(torch.randn(M, N, generator=g, device="cuda"))
        y = dense(M, N, t, pad, offset)
        ws = polyq_lib.fp4_workspace()
        polyq_lib.fp4_linear(x, w, y=y, residual=res, workspace=ws)
        ref = prod + res.double()
        # as fp4_util.sum_bound, with up to 100 parts of a shared tile
        bound = (2 * (-(-K // 64)) + 110) * U32 * (S + res.double().abs()) * 1.01 + ref.abs() * half_step(t) + tiny(t)
        off = (y.double() - ref).abs() - bound
        assert bool(torch.isfinite(y).all()) and float(off.max()) <= 0, (t, pad, float(off.max()))
        if pad:  # what lies between the rows is not touched
            assert bool(torch.isnan(y.as_strided((M - 1, pad), (N + pad, 1), offset + N)).all())
        polyq_lib.fp4_linear(x, w, y=res, residual=res, workspace=ws)
        assert torch.equal(res, y)
        assert polyq_lib.workspace_status(ws) == 0 and int(ws[:polyq_lib.FP4_WORKSPACE_ZERO].max()) == 0


@pytest.mark.parametrize("fmt", [MX, NV])
@pytest.mark.parametrize("M,N,pad", [(1, 256, 0), (8, 256, 0), (8, 100, 3), (100, 256, 0), (2304, 256, 0), (2304, 100, 3)])
def test_chained(polyq_lib, fmt, M, N, pad):
    """A residual stream: the same buffer added to by every call, or two in turn,
    quantised between the calls, in a graph whose launches overlap and whose
    replays use the same addresses; as one call at a time gives it."""
    g = torch.Generator("cuda").manual_seed(M + N)
    n = 24
    w = [_q(polyq_lib, g, N, N, fmt, N ** -0.5) for _ in range(3)]
    start = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    bufs = [dense(M, N, torch.bfloat16, pad) for _ in range(2)]
    q = polyq_lib.Fp4Tensor.empty(M, N, fmt, 1.0 if fmt == MX else 2.0 ** -8)
    ws = polyq_lib.fp4_workspace()

    def run(turns, synchronize=False):
        bufs[0].copy_(start)
        for i in range(n):
            src, dst = bufs[i % turns], bufs[(i + 1) % turns]
            if i % 3 == 0:
                polyq_lib.fp4_quantize(src, out=q)
            polyq_lib.fp4_linear(q, w[i % 3], y=dst, residual=src, workspace=ws)
            if synchronize:
                torch.cuda.synchronize()

    for turns in (1, 2):  # n is even: the result is in the first buffer
        run(turns, True)
        want = bufs[0].clone()
        assert bool(torch.isfinite(want).all())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(turns)
        for _ in range(5):
            for b in bufs:
                b.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(bufs[0], want)
        run(turns)
        assert torch.equal(bufs[0], want)
