"""GPU tests of adapters beside the mixed-width layers: on the same x and onto the same y, decoding
(linear_gemv, captured in a graph too) and on prompts (linear_gemm), with the layer's rows in their
own order and permuted."""
import numpy as np
import pytest
import torch

from oracle import polyq_oracle as O
from tests import finetune_util as F
from tests.gpu_util import check_tolerance, make_case, oracle_layer
from tests.test_gpu_adapters import within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,segments,ids", [(1, [0, 1], [2]), (4, [0, 1, 3, 4], [0, -1, 1]),
                                               (100, [0, 40, 100], [1, 0])])
@pytest.mark.parametrize("permuted", [False, True])
def test_beside_a_mixed_width_layer(polyq_lib, rows, segments, ids, permuted):
    """x is in the order of the layer's columns, whatever its clustering; b's rows are in that of its y:
    its own, or that which permute_rows has given it."""
    N, K, R, n = 300, 1500, 16, 3
    W, act, bits, xb, x64 = make_case(N, K, 3.0, 12, True, rows)
    host = polyq_lib.HostLayer.pack(W, act, 3.0, forced_bits=bits)
    order = np.random.default_rng(1).permutation(N) if permuted else np.arange(N)
    if permuted:
        host.permute_rows(order)
    layer = polyq_lib.DeviceLayer(host, "cuda")
    linear = polyq_lib.linear_gemv if rows <= 4 else polyq_lib.linear_gemm
    x = torch.from_numpy(xb.view(np.int16)).cuda().view(torch.bfloat16)
    g = torch.Generator("cuda").manual_seed(3)
    a = torch.zeros(n, R, K + 4, dtype=torch.bfloat16, device="cuda")[:, :, :K]  # (rows on 16 bytes)
    a.copy_(torch.randn(n, R, K, generator=g, device="cuda") * 0.02)
    b_own = (torch.randn(n, N, R, generator=g, device="cuda") * 0.1).bfloat16()  # of the channels' own order
    b = b_own[:, torch.from_numpy(order).cuda()].contiguous()
    off, who = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (segments, ids))
    ws = polyq_lib.adapters_workspace(rows, R)
    lws = torch.zeros(polyq_lib.gemv_workspace_bytes(layer, rows) if rows <= 4 else
                      polyq_lib.gemm_workspace_bytes(layer, rows), dtype=torch.uint8, device="cuda")
    base, y = (torch.empty(rows, N, device="cuda") for _ in range(2))

    def call():
        linear(layer, x, y, workspace=lws)
        base.copy_(y)  # (whose last bits differ from call to call: its parts are added as they come)
        polyq_lib.adapters_forward(x, a, b, off, who, residual=y, y=y, workspace=ws)

    plain = O.linear(oracle_layer(W, act, 3.0, bits), x64)
    for s0, s1, i in zip(segments, segments[1:], ids):
        if i >= 0:
            v = x64[s0:s1] @ a[i].double().cpu().numpy().T
            plain[s0:s1] += v @ b_own[i].double().cpu().numpy().T

    def look():
        torch.cuda.synchronize()
        ref = F.adapters(x, a, b, segments, ids, [1.0] * n, [R] * n, base.double(), out=torch.float32)
        within(y, *ref[0], "y")
        check_tolerance(y.cpu().numpy(), plain[:, order], x64, K)

    call()
    look()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(2):
        y.fill_(float("nan"))
        graph.replay()
        look()
