"""Performance cases of the 4-bit floating-point operators and the gated feed-forward block.

Each case is one pass through an operator of ``paper_2607_14618_gb300.polyq`` as a user's program
makes it: quantising a tensor to microscaled 4-bit floating point and back (``fp4_quantize``,
``fp4_dequantize``), a product of two quantised tensors (``fp4_linear``), a gated feed-forward
block on quantised operands (``fp4_ffn``), the whole quantised block of a decoder layer, or a
training step's forward and backward through the gated block in 16 bits (``ffn_forward``,
``ffn_backward``).  ``listed()`` names the standing cases, ``draw()`` gives others of the same
ranges, ``prepare()`` makes the inputs, quantised weights and buffers that a program keeps,
``run()`` is the timed pass (plain torch operations, or with ``own`` the framework's operators)
and ``exact()`` the same result in 64 bits.

Inputs follow the synthetic recipe of ``synth.py`` on the GPU: weights N(0, 0.02^2) with 1% of the
columns x10, activation magnitudes lognormal(0, 1) with 1% of the channels x20, activations
magnitude * N(0, 1), normalised to unit mean square per row as behind an RMSNorm.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = {"mx": 32, "nv": 16}  # elements that share a scale


def listed():
    """The standing cases."""
    return [
        # One token's hidden state through the quantiser: launches and the host path count.
        {"name": "quant_b1_mx", "kind": "quant", "rows": 1, "K": 5120, "fmt": "mx", "x": "bf16"},
        # A strided slice of a wider buffer with a last block of a few elements.
        {"name": "quant_odd_nv", "kind": "quant", "rows": 777, "K": 5003, "fmt": "nv", "x": "f16"},
        # Fake quantisation of a fp32 master weight in a training step.
        {"name": "quant_gate_f32_nv", "kind": "quant", "rows": 13824, "K": 5120, "fmt": "nv",
         "x": "f32"},
        # The down projection of one token, with the residual stream added.
        {"name": "linear_b1_down_mx", "kind": "linear", "M": 1, "N": 5120, "K": 13824, "fmt": "mx",
         "y": "f32", "res": True},
        # A batch of sequences decoded together on the widest layer.
        {"name": "linear_m48_gate_nv", "kind": "linear", "M": 48, "N": 13824, "K": 5120,
         "fmt": "nv", "y": "bf16", "res": False},
        # Ragged in every dimension.
        {"name": "linear_odd_m203_mx", "kind": "linear", "M": 203, "N": 4099, "K": 2501,
         "fmt": "mx", "y": "f16", "res": False},
        # A long prompt: the largest product.
        {"name": "linear_m8192_down_nv", "kind": "linear", "M": 8192, "N": 5120, "K": 13824,
         "fmt": "nv", "y": "bf16", "res": True},
        # Gate and up of one token.
        {"name": "ffn4_b1_mx", "kind": "ffn4", "M": 1, "F": 13824, "K": 5120, "fmt": "mx",
         "y": "bf16"},
        # Gate and up of a prefill chunk.
        {"name": "ffn4_m2048_nv", "kind": "ffn4", "M": 2048, "F": 13824, "K": 5120, "fmt": "nv",
         "y": "bf16"},
        # The whole block of a short prompt: activations quantised, gate and up with a quantised
        # output, down with the residual.
        {"name": "mlp4_m512_mx", "kind": "mlp4", "M": 512, "F": 13824, "K": 5120, "fmt": "mx"},
        # A small training step of odd sizes.
        {"name": "train_odd_t301_f16", "kind": "train", "T": 301, "F": 2731, "K": 1000, "x": "f16"},
        # A training step on the widest block: the largest.
        {"name": "train_t4096_bf16", "kind": "train", "T": 4096, "F": 13824, "K": 5120,
         "x": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(("quant", "linear", "linear", "ffn4", "mlp4", "train"))
    fmt = rng.choice(("mx", "nv"))
    rows = _log_int(rng, 1, 8192 if kind in ("quant", "linear") else 4096)
    n, k = _log_int(rng, 128, 16384), _log_int(rng, 128, 16384)
    if rng.random() < 0.6:  # most layers are multiples of 64; the others keep their odd sizes
        n, k = max(128, n // 64 * 64), max(128, k // 64 * 64)
    while n * k > 13824 * 5120:
        n = max(128, n // 2)
    if kind == "quant":
        return {"kind": kind, "rows": rows, "K": k, "fmt": fmt, "x": rng.choice(("f32", "bf16", "f16"))}
    if kind == "linear":
        return {"kind": kind, "M": rows, "N": n, "K": k, "fmt": fmt,
                "y": rng.choice(("f32", "bf16", "f16")), "res": rng.random() < 0.5}
    if kind == "ffn4":
        return {"kind": kind, "M": rows, "F": n, "K": k, "fmt": fmt,
                "y": rng.choice(("bf16", "f16"))}
    if kind == "mlp4":
        return {"kind": kind, "M": rows, "F": n, "K": k, "fmt": fmt}
    # 16-bit rows start on 16 bytes: K is a multiple of 8
    return {"kind": kind, "T": rows, "F": n, "K": max(128, k // 8 * 8),
            "x": rng.choice(("bf16", "f16"))}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(DEV).manual_seed(int(seed))


def _weights(g, N, K):
    """fp32 weights [N][K]."""
    W = torch.randn(N, K, generator=g, device=DEV).mul_(0.02)
    W[:, torch.randperm(K, generator=g, device=DEV)[:round(0.01 * K)]] *= 10.0
    return W


def _acts(g, rows, K):
    """fp32 activations [rows][K] with outlier channels."""
    m = torch.exp(torch.randn(K, generator=g, device=DEV))
    m[torch.randperm(K, generator=g, device=DEV)[:round(0.01 * K)]] *= 20.0
    x = m * torch.randn(rows, K, generator=g, device=DEV)
    return x.div_(x.square().mean(1, keepdim=True).sqrt_())


def _tensor_scale(fmt, amax):
    """The power of two that brings the largest block scale of an NV tensor under e4m3's 448."""
    return 1.0 if fmt == "mx" or amax == 0 else 2.0 ** math.ceil(math.log2(amax / (6 * 448)))


def _raw(case, seed):
    """The case's unquantised inputs."""
    g, kind = _gen(seed), case["kind"]
    if kind == "quant":
        wider = 13 if case["K"] % 64 else 0  # odd widths are rows of a wider buffer
        x = (_weights if case["x"] == "f32" else _acts)(g, case["rows"], case["K"] + wider)
        return {"x": x.to(TYPES[case["x"]])[:, :case["K"]]}
    if kind == "linear":
        d = {"x": _acts(g, case["M"], case["K"]).to(torch.bfloat16), "w": _weights(g, case["N"], case["K"])}
        if case["res"]:
            d["res"] = torch.randn(case["M"], case["N"], generator=g, device=DEV).to(TYPES[case["y"]])
        return d
    rows, t = (case["T"], TYPES[case["x"]]) if kind == "train" else (case["M"], torch.bfloat16)
    F, K = case["F"], case["K"]
    d = {"x": _acts(g, rows, K).to(t), "gate": _weights(g, F, K), "up": _weights(g, F, K)}
    if kind == "train":
        d["gate"], d["up"] = d["gate"].to(t), d["up"].to(t)
        d["dh"] = torch.randn(rows, F, generator=g, device=DEV).to(t)
    if kind == "mlp4":
        d["down"] = _weights(g, K, F)
        d["res"] = torch.randn(rows, K, generator=g, device=DEV).to(torch.bfloat16)
        d["g_h"] = _tensor_scale(case["fmt"], 256.0)  # calibrated range of the block's middle
    return d


def prepare(case, seed):
    """Inputs, quantised tensors and the buffers of a program that repeats the call."""
    kind, d = case["kind"], _raw(case, seed)
    st = {"case": case, **d}
    fmt = case.get("fmt")
    names = {"quant": (), "linear": ("x", "w"), "ffn4": ("x", "gate", "up"),
             "mlp4": ("gate", "up", "down"), "train": ()}[kind]
    scales = {n: _tensor_scale(fmt, float(d[n].abs().max())) for n in names}
    if kind in ("quant", "mlp4"):
        scales["x"] = _tensor_scale(fmt, float(d["x"].abs().max()))
    st["g"] = scales
    if own:
        from paper_2607_14618_gb300 import polyq
        f = polyq.FP4_MX if fmt == "mx" else polyq.FP4_NV
        for n in names:
            st[n] = polyq.fp4_quantize(d[n], f, scales[n])
        if kind == "quant":
            st["q"] = polyq.Fp4Tensor.empty(case["rows"], case["K"], f, scales["x"], device=DEV)
            st["v"] = torch.empty(case["rows"], case["K"], dtype=torch.bfloat16, device=DEV)
        elif kind == "linear":
            st["ws"] = polyq.fp4_workspace(DEV)
            st["y"] = torch.empty(case["M"], case["N"], dtype=TYPES[case["y"]], device=DEV)
        elif kind == "ffn4":
            st["ws"] = polyq.fp4_workspace(DEV)
            st["y"] = torch.empty(case["M"], case["F"], dtype=TYPES[case["y"]], device=DEV)
        elif kind == "mlp4":
            st["ws"] = polyq.fp4_workspace(DEV)
            st["xq"] = polyq.Fp4Tensor.empty(case["M"], case["K"], f, scales["x"], device=DEV)
            st["hq"] = polyq.Fp4Tensor.empty(case["M"], case["F"], f, d["g_h"], device=DEV)
            st["y"] = torch.empty(case["M"], case["K"], dtype=torch.bfloat16, device=DEV)
        else:
            st["ws"] = polyq.ffn_workspace(case["T"], case["F"], case["K"], DEV)
            st["saved"] = polyq.ffn_saved(case["T"], case["F"], d["x"].dtype, DEV)
            st["h"] = torch.empty_like(d["dh"])
            st["dx"], st["dgate"], st["dup"] = (torch.empty_like(d[n]) for n in ("x", "gate", "up"))
    else:
        for n in names:
            st[n] = _quantise(d[n], fmt, scales[n])
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _quantise(x, fmt, g):
    """Codes 0..15 (sign in bit 3) uint8 [rows][K] and block scales fp32 [rows][blocks]."""
    rows, K = x.shape
    B = BLOCK[fmt]
    t = torch.nn.functional.pad(x.float(), (0, -K % B)).reshape(rows, -1, B)
    if fmt == "mx":
        amax = t.abs().amax(2)
        e = (torch.frexp(amax).exponent - 3).clamp(-127, 127)  # floor(log2(amax)) - 2
        s = torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.zeros_like(amax))
    else:
        t = t / g
        s = (t.abs().amax(2) / 6).clamp(max=448).to(torch.float8_e4m3fn).float()
    a = t.abs() / torch.where(s > 0, s, torch.full_like(s, math.inf))[:, :, None]
    # ties to the even code: borders below an even code belong to it, the others to the lower one
    q = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5)
         + (a > 5.0))
    q = q + 8 * (t < 0)
    return q.reshape(rows, -1)[:, :K], s, g


def _values(q, fmt):
    """fp32 values of codes and scales."""
    codes, s, g = q
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    v = torch.cat((grid, -grid))[codes.int()]
    return v * (s * g).repeat_interleave(BLOCK[fmt], 1)[:, :codes.shape[1]]


def _plain(st):
    case = st["case"]
    kind, fmt = case["kind"], case.get("fmt")
    if kind == "quant":
        return _values(_quantise(st["x"], fmt, st["g"]["x"]), fmt).to(torch.bfloat16)
    if kind == "linear":
        y = _values(st["x"], fmt) @ _values(st["w"], fmt).T
        return (y + st["res"].float() if case["res"] else y).to(TYPES[case["y"]])
    if kind in ("ffn4", "mlp4"):
        x = _values(st["x"] if kind == "ffn4" else _quantise(st["x"], fmt, st["g"]["x"]), fmt)
        a = x @ _values(st["gate"], fmt).T
        h = a / (1 + torch.exp(-a)) * (x @ _values(st["up"], fmt).T)
        if kind == "ffn4":
            return h.to(TYPES[case["y"]])
        y = _values(_quantise(h, fmt, st["g_h"]), fmt) @ _values(st["down"], fmt).T
        return (st["res"].float() + y).to(torch.bfloat16)
    x, gate, up, dh = (st[n].float() for n in ("x", "gate", "up", "dh"))
    a, u = x @ gate.T, x @ up.T
    s = 1 / (1 + torch.exp(-a))
    da, du = dh * u * s * (1 + a * (1 - s)), dh * a * s
    t = st["x"].dtype
    return {"h": (a * s * u).to(t), "dx": (da @ gate + du @ up).to(t),
            "dgate": (da.T @ x).to(t), "dup": (du.T @ x).to(t)}


def run(st):
    """One pass through the case's operator."""
    if not own:
        return _plain(st)
    from paper_2607_14618_gb300 import polyq
    case = st["case"]
    kind = case["kind"]
    if kind == "quant":
        q = polyq.fp4_quantize(st["x"], out=st["q"])
        return polyq.fp4_dequantize(q, out=st["v"])
    if kind == "linear":
        return polyq.fp4_linear(st["x"], st["w"], y=st["y"], residual=st.get("res"),
                                workspace=st["ws"])
    if kind == "ffn4":
        return polyq.fp4_ffn(st["x"], st["gate"], st["up"], st["y"], workspace=st["ws"])
    if kind == "mlp4":
        polyq.fp4_quantize(st["x"], out=st["xq"])
        polyq.fp4_ffn(st["xq"], st["gate"], st["up"], st["hq"], workspace=st["ws"])
        return polyq.fp4_linear(st["hq"], st["down"], y=st["y"], residual=st["res"],
                                workspace=st["ws"])
    polyq.ffn_forward(st["x"], st["gate"], st["up"], h=st["h"], saved=st["saved"],
                      workspace=st["ws"])
    polyq.ffn_backward(st["x"], st["gate"], st["up"], st["saved"], st["dh"], dx=st["dx"],
                       dgate=st["dgate"], dup=st["dup"], workspace=st["ws"])
    return {n: st[n] for n in ("h", "dx", "dgate", "dup")}


# ---------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    """Operands in and results out once; two operations a multiplication and addition.  A quantised
    tensor is half a byte an element and a byte a block.  A training step reads x, the weights and
    dh, and writes h and the gradients of x and the weights."""
    kind = case["kind"]

    def q(rows, K):
        return rows * (0.5 * K + math.ceil(K / BLOCK[case["fmt"]]))

    if kind == "quant":
        n = case["rows"] * case["K"]
        return {"bytes": n * BYTES[case["x"]] + 2 * q(case["rows"], case["K"]) + 2 * n, "flops": 4.0 * n}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        out = M * N * BYTES[case["y"]]
        return {"bytes": q(M, K) + q(N, K) + out * (2 if case["res"] else 1), "flops": 2.0 * M * N * K}
    if kind == "ffn4":
        M, F, K = case["M"], case["F"], case["K"]
        return {"bytes": q(M, K) + 2 * q(F, K) + M * F * BYTES[case["y"]], "flops": 4.0 * M * F * K}
    if kind == "mlp4":
        M, F, K = case["M"], case["F"], case["K"]
        return {"bytes": 2.0 * M * K + 2 * q(F, K) + q(K, F) + 4.0 * M * K, "flops": 6.0 * M * F * K}
    T, F, K = case["T"], case["F"], case["K"]
    return {"bytes": 2.0 * (2 * T * K + 4 * F * K + 2 * T * F), "flops": 12.0 * T * F * K}


_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_values(x, fmt, g):
    """The values of a quantised tensor in 64 bits, found as the nearest grid value of the scaled
    element (of two equally near, the one with the even code)."""
    B, (rows, K) = BLOCK[fmt], x.shape
    n = -(-K // B)
    t = torch.zeros(rows, n * B, dtype=torch.float64, device=x.device)
    t[:, :K] = x.double() / g
    t = t.view(rows, n, B)
    top = t.abs().amax(2, keepdim=True)
    if fmt == "mx":
        e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
        e = e + (torch.exp2(e + 1) <= top).double() - (torch.exp2(e) > top).double()  # log2 at a border
        s = torch.exp2((e - 2).clamp(-127, 127))
    else:
        v = top / 6
        e = torch.floor(torch.log2(v.clamp(min=2.0 ** -20)))
        step = torch.exp2(e.clamp(min=-6) - 3)  # e4m3: three bits behind the leading one
        s = (torch.round(v / step) * step).clamp(max=448)
        s = torch.where(s > 0, s, torch.ones_like(s) * 1e300)
    a = t.abs() / s
    lower = torch.zeros_like(a)
    out = torch.zeros_like(a)
    for i, (lo, hi) in enumerate(zip(_GRID, _GRID[1:])):
        half = (lo + hi) / 2
        up = (a > half) | ((a == half) if i % 2 else torch.zeros_like(a, dtype=torch.bool))
        lower = torch.where(up, torch.full_like(a, hi), torch.full_like(a, lo))
        out = torch.where(a >= lo, lower, out)
    out = torch.where(a >= 6, torch.full_like(a, 6.0), out)
    s = torch.where(s > 1e299, torch.zeros_like(s), s)
    return (torch.sign(t) * out * s * g).view(rows, n * B)[:, :K]


def exact(case, seed):
    """The outputs of the case in 64 bits, from the definitions."""
    kind, fmt, d = case["kind"], case.get("fmt"), _raw(case, seed)

    def q(name):
        return _exact_values(d[name], fmt, _tensor_scale(fmt, float(d[name].abs().max())))

    if kind == "quant":
        return q("x")
    if kind == "linear":
        y = torch.matmul(q("x"), q("w").t())
        return y + d["res"].double() if case["res"] else y
    if kind != "train":
        x = q("x")
        a = torch.matmul(x, q("gate").t())
        h = a * torch.sigmoid(a) * torch.matmul(x, q("up").t())
        if kind == "ffn4":
            return h
        return d["res"].double() + torch.matmul(_exact_values(h, fmt, d["g_h"]), q("down").t())
    x, gate, up, dh = (d[n].double() for n in ("x", "gate", "up", "dh"))
    a, u = torch.matmul(x, gate.t()), torch.matmul(x, up.t())
    s = torch.sigmoid(a)
    du, da = dh * (a * s), dh * u * (s + a * s * (1 - s))
    return {"h": a * s * u, "dx": torch.matmul(da, gate) + torch.matmul(du, up),
            "dgate": torch.matmul(da.t(), x), "dup": torch.matmul(du.t(), x)}
