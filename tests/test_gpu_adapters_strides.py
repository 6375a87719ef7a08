"""GPU tests of adapters whose matrices lie otherwise than one after another: a and b of each adapter
in one buffer (the distance to the next is no multiple of a row's), one matrix for all, the adapters' rows
in turn, every second one; with segments of few and of many rows."""
import pytest
import torch

from tests import finetune_util as F
from tests.test_gpu_adapters import segments, within

pytestmark = pytest.mark.gpu


def matrices(kind, n, R, K, N, dtype):
    """a [n][R][K] and b [n][N][R]."""
    g = torch.Generator("cuda").manual_seed(5)
    a = (torch.randn(n, R, K, generator=g, device="cuda") * K ** -0.5).to(dtype)
    b = (torch.randn(n, N, R, generator=g, device="cuda") * 0.1).to(dtype)
    if kind == "packed":
        each = R * K + N * R + 8
        buf = torch.full((n * each,), float("nan"), dtype=dtype, device="cuda")
        pa = buf.as_strided((n, R, K), (each, K, 1))
        pb = buf[R * K:].as_strided((n, N, R), (each, R, 1))
        assert each % K and each % R
        return pa.copy_(a), pb.copy_(b)
    if kind == "shared a":
        return a[:1].expand(n, R, K), b
    if kind == "shared b":
        return a, b[:1].expand(n, N, R)
    if kind == "rows in turn":  # row j of every adapter, then row j + 1
        return (a.transpose(0, 1).contiguous().transpose(0, 1), b.transpose(0, 1).contiguous().transpose(0, 1))
    wide = [torch.full((2 * n, *t.shape[1:]), float("nan"), dtype=dtype, device="cuda") for t in (a, b)]
    return [w[1::2].copy_(t) for w, t in zip(wide, (a, b))]


@pytest.mark.parametrize("kind", ["packed", "shared a", "shared b", "rows in turn", "every second"])
@pytest.mark.parametrize("lengths,ids", [([3, 1, 2], [2, 0, 1]), ([70, 50, 129], [1, 2, 1]), ([600, 300], [2, 1])])
@pytest.mark.parametrize("R", [16, 64])
def test_places_of_the_matrices(polyq_lib, kind, lengths, ids, R):
    n, K, N, T = 3, 520, 264, sum(lengths)
    for dtype in (torch.bfloat16, torch.float16):
        g = torch.Generator("cuda").manual_seed(6)
        x, dy = (torch.randn(T, c, generator=g, device="cuda").to(dtype) for c in (K, N))
        a, b = matrices(kind, n, R, K, N, dtype)
        off, d_off = segments(lengths)
        d_ids = torch.tensor(ids, dtype=torch.int32, device="cuda")
        saved, ws = polyq_lib.adapters_saved(T, R), polyq_lib.adapters_workspace(T, R)
        y = polyq_lib.adapters_forward(x, a, b, d_off, d_ids, dtype=torch.float32, saved=saved, workspace=ws)
        da, db = (torch.empty(s, device="cuda") for s in ((n, R, K), (n, N, R)))
        dx = torch.empty(T, K, device="cuda")
        polyq_lib.adapters_backward(x, a, b, saved, dy, d_off, d_ids, dx=dx, da=da, db=db, workspace=ws)
        zero = [torch.zeros(T, c, dtype=torch.float64, device="cuda") for c in (N, K)]
        ref = F.adapters(x, a, b, off, ids, [1.0] * n, [R] * n, zero[0], dy, zero[1], *[torch.float32] * 3)
        for got, want, what in zip((y, dx, da, db), ref, ("y", "dx", "da", "db")):
            within(got, *want, what)
        assert polyq_lib.workspace_status(ws) == 0
        if kind not in ("packed", "rows in turn"):  # (which are copied in another way)
            again = polyq_lib.adapters_forward(x, a.contiguous(), b.contiguous(), d_off, d_ids, dtype=torch.float32)
            assert torch.equal(y, again)
