"""GPU tests of the adapters' gradients over thousands of rows of one adapter."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -23


@pytest.mark.parametrize("dtype,run", [(torch.bfloat16, 128), (torch.float16, 64)])
def test_sums_start_anew(polyq_lib, dtype, run):
    """Sums of positive numbers over 8192 rows stay near fp32's own roundings.

    a and b pick channels, so that v and dv are x's and dy's own 16-bit numbers: their parts, products
    and second halves are exact, and what is left are the sums.  The tensor cores cut a running sum off
    by two units (2^-23 of it) at most for every 16 products; sums that start anew every `run` rows reach
    S_run in run / 16 steps, which is (run / 16 + 1) units of S_run, the same part of the total.  Each is
    added in fp32: half a unit of what has been summed so far, (8192 / run + 1) / 4 units of the total;
    three more are for fp16's scale and the result.  A sum that never starts anew is cut off 512 times,
    which at half a unit each is 128 units.

    K and N make for enough blocks that none shares its rows with others (304 and more, two an SM)."""
    T, K, N, R = 8192, 1024, 38912, 16
    g = torch.Generator("cuda").manual_seed(2)
    x, dy = ((torch.rand(T, c, generator=g, device="cuda") * 0.5 + 0.5).to(dtype) for c in (K, N))
    a, b = torch.zeros(1, R, K, dtype=dtype, device="cuda"), torch.zeros(1, N, R, dtype=dtype, device="cuda")
    j = torch.arange(R, device="cuda")
    ka, nb = j * 60 + 3, j * 2000 + 7  # the channels that are v and dv
    a[0, j, ka], b[0, nb, j] = 1, 1
    off, ids = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, T], [0]))
    saved = polyq_lib.adapters_saved(T, R)
    polyq_lib.adapters_forward(x, a, b, off, ids, saved=saved)
    assert torch.equal(saved, x[:, ka].float())
    da, db = torch.empty(1, R, K, device="cuda"), torch.empty(1, N, R, device="cuda")
    polyq_lib.adapters_backward(x, a, b, saved, dy, off, ids, need_dx=False, da=da, db=db)
    bound = ((run / 16 + 1) + (T / run + 1) / 4 + 3) * U32
    for got, want, what in ((da[0], dy[:, nb].double().T @ x.double(), "da"),
                            (db[0], dy.double().T @ x[:, ka].double(), "db")):
        off_by = ((got.double() - want).abs() / want).max().item()
        print(what, off_by / U32, bound / U32)
        assert off_by <= bound, (what, off_by / U32, bound / U32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R", [16, 40, 128])
@pytest.mark.parametrize("rows", [(2100,), (9000,), (5000, 1, 0), (1100, 1300, 1030)])
def test_shared_rows(polyq_lib, dtype, R, rows):
    """Blocks that share the rows of an adapter (two, four and eight of them, some without a row) add
    up to what 64 bits give, and to the same bits again."""
    n, K, N, T = len(rows), 136, 264, sum(rows)
    g = torch.Generator("cuda").manual_seed(4)
    x, dy = (torch.randn(T, c, generator=g, device="cuda").to(dtype) for c in (K, N))
    a, b = ((torch.randn(n, *s, generator=g, device="cuda") * 0.1).to(dtype) for s in ((R, K), (N, R)))
    cuts = [0]
    for r in rows:
        cuts.append(cuts[-1] + r)
    off, ids = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (cuts, list(range(n))))
    saved = polyq_lib.adapters_saved(T, R)
    polyq_lib.adapters_forward(x, a, b, off, ids, saved=saved)
    out = []
    for _ in range(2):
        da, db = (torch.full((n, *s), float("nan"), device="cuda") for s in ((R, K), (N, R)))
        polyq_lib.adapters_backward(x, a, b, saved, dy, off, ids, need_dx=False, da=da, db=db)
        out.append((da, db))
    assert all(torch.equal(p, q) for p, q in zip(*out))
    for i in range(n):
        s = slice(cuts[i], cuts[i + 1])
        X, D, A, B = x[s].double(), dy[s].double(), a[i].double(), b[i].double()
        v, dv = X @ A.T, D @ B
        for got, want, size in ((out[0][0][i], dv.T @ X, dv.abs().T @ X.abs()),
                                (out[0][1][i], D.T @ v, D.abs().T @ v.abs())):
            # what is lost of v and dv (2^-17 in bf16, 2^-22 in fp16), their own sums (17 steps of two
            # units), a run of both halves (16 steps), the runs' sum and that of eight blocks
            rel = (2.0 ** -17 if dtype == torch.bfloat16 else 2.0 ** -22) + (2 * 17 + 20 + len(X) / 256 + 16) * U32
            assert ((got.double() - want).abs() <= rel * size + 1e-30).all()
