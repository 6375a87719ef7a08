"""Performance cases of the operators that fine-tune a quantised model and serve the result.

Each case is one pass through an operator of ``paper_2607_14618_gb300.polyq`` as a user's program
makes it: layer norm (with or without the mean) and its backward pass (``layernorm_forward``,
``layernorm_backward``), an AdamW step over many tensors with states in 32 or 8 bits
(``AdamW.step``, ``AdamState.values``), or low-rank adapters of many requests beside a projection
whose result they add to (``adapters_forward``), with their gradients in training
(``adapters_backward``).  ``listed()`` names the standing cases, ``draw()`` gives others of the
same ranges, ``prepare()`` makes the inputs and what a program keeps, ``run()`` is the timed pass
(plain torch operations, or with ``own`` the framework's operators) and ``exact()`` the same result
in 64 bits.

Activations follow the synthetic recipe of ``synth.py``: magnitudes lognormal(0, 1) with 1% of the
channels x20, times N(0, 1).  Sizes are those of the layers that ``bench.py`` and ``synth.py`` use
(5120 x 13824) and generic ones.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "none": 0}
EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY = 2e-4, 0.9, 0.95, 1e-8, 0.1
BLOCK = 256  # elements of an 8-bit state that share a scale


def listed():
    """The standing cases."""
    return [
        # One token's residual stream in fp32 through the norm before a projection: latency.
        {"name": "norm_b1", "kind": "norm", "rows": 1, "K": 5120, "x": "f32", "y": "bf16",
         "center": False, "bias": False, "train": False, "res": False},
        # A long prompt through a layer norm with a bias.
        {"name": "norm_prompt", "kind": "norm", "rows": 8192, "K": 5120, "x": "bf16", "y": "bf16",
         "center": True, "bias": True, "train": False, "res": False},
        # A training step of odd sizes: contiguous rows that start on 2 bytes.
        {"name": "norm_train_odd", "kind": "norm", "rows": 777, "K": 5003, "x": "f16", "y": "f16",
         "center": True, "bias": True, "train": True, "res": False},
        # A training step with the residual stream's own gradient added to dx.
        {"name": "norm_train", "kind": "norm", "rows": 8192, "K": 5120, "x": "bf16", "y": "bf16",
         "center": False, "bias": False, "train": True, "res": True},
        # The norms' gains of 40 layers: many small vectors.
        {"name": "adamw8_gains", "kind": "adamw", "tensors": 81, "n": 5120, "p": "f32",
         "g": "f32", "copy": "none", "bits": 8},
        # The adapters of 40 layers, seven projections each (rank 16): many middling tensors.
        {"name": "adamw32_adapters", "kind": "adamw", "tensors": 560, "n": 110592, "p": "f32",
         "g": "bf16", "copy": "bf16", "bits": 32},
        # A gated block's three matrices, fp32 master weights and the bf16 weights made of them.
        {"name": "adamw32_block", "kind": "adamw", "tensors": 3, "n": 70778880, "p": "f32",
         "g": "bf16", "copy": "bf16", "bits": 32},
        # The same with states in 8 bits (the values that they stand for written out as well).
        {"name": "adamw8_block", "kind": "adamw", "tensors": 3, "n": 70778880, "p": "f32",
         "g": "bf16", "copy": "bf16", "bits": 8},
        # One token of one request: latency.
        {"name": "adapters_b1", "kind": "adapters", "T": 1, "K": 5120, "N": 13824, "R": 16,
         "segments": 1, "adapters": 8, "bare": 0, "x": "bf16", "y": "f32", "train": False},
        # 48 requests decoded together, each with an adapter of its own.
        {"name": "adapters_decode48", "kind": "adapters", "T": 48, "K": 5120, "N": 13824, "R": 64,
         "segments": 48, "adapters": 96, "bare": 0, "x": "f16", "y": "f16", "train": False},
        # Prompts of ragged lengths, two requests without an adapter, ranks up to 32.
        {"name": "adapters_prompts", "kind": "adapters", "T": 6007, "K": 13824, "N": 5120, "R": 32,
         "segments": 13, "adapters": 7, "bare": 2, "x": "bf16", "y": "bf16", "train": False},
        # A training step of two adapters on the widest projection.
        {"name": "adapters_train", "kind": "adapters", "T": 4096, "K": 5120, "N": 13824, "R": 64,
         "segments": 4, "adapters": 2, "bare": 0, "x": "bf16", "y": "bf16", "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(("norm", "adamw", "adapters"))
    if kind == "norm":
        x = rng.choice(("f32", "bf16", "f16"))
        K = _log_int(rng, 64, 16384)
        if rng.random() < 0.6:  # most widths are multiples of 64; the others keep their odd sizes
            K = max(64, K // 64 * 64)
        rows = min(_log_int(rng, 1, 16384), 8192 * 5120 // K)
        center = rng.random() < 0.5
        return {"kind": kind, "rows": rows, "K": K, "x": x, "y": rng.choice((x, "bf16")),
                "center": center, "bias": center and rng.random() < 0.7,
                "train": rng.random() < 0.6, "res": rng.random() < 0.5}
    if kind == "adamw":
        tensors = _log_int(rng, 1, 700)
        n = _log_int(rng, 1, 2.0e8 / tensors)
        p = rng.choice(("f32", "f32", "bf16", "f16"))
        return {"kind": kind, "tensors": tensors, "n": n, "p": p,
                "g": rng.choice(("f32", "bf16", "f16")) if p == "f32" else rng.choice((p, "f32")),
                "copy": rng.choice(("none", "bf16", "f16")) if p == "f32" else "none",
                "bits": rng.choice((8, 32))}
    train = rng.random() < 0.4
    T = _log_int(rng, 1, 4096 if train else 8192)
    segments = _log_int(rng, 1, min(T, 64))
    # rows of 16-bit operands start on 16 bytes: K is a multiple of 8; N may be odd
    N = _log_int(rng, 256, 13824)
    return {"kind": kind, "T": T, "K": _log_int(rng, 256, 13824) // 8 * 8,
            "N": N if rng.random() < 0.3 else N // 64 * 64,
            "R": rng.choice((8, 16, 24, 32, 64)), "segments": segments,
            "adapters": _log_int(rng, 1, min(32, 2 * segments)),
            "bare": rng.choice((0, 0, 1)) if segments > 1 else 0,
            "x": rng.choice(("bf16", "f16")), "y": rng.choice(("f32", "x")), "train": train}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(DEV).manual_seed(int(seed))


def _acts(g, rows, K):
    """fp32 activations [rows][K] with outlier channels, of mean square 1 over all rows."""
    m = torch.exp(torch.randn(K, generator=g, device=DEV))
    m[torch.randperm(K, generator=g, device=DEV)[:round(0.01 * K)]] *= 20.0
    x = torch.randn(rows, K, generator=g, device=DEV).mul_(m)
    return x.div_(x.square().mean().sqrt_())


def _norm_inputs(case, seed):
    g = _gen(seed)
    rows, K, tx, ty = case["rows"], case["K"], TYPES[case["x"]], TYPES[case["y"]]
    d = {"x": (_acts(g, rows, K) * 2 + 0.3).to(tx),
         "w": 1 + 0.1 * torch.randn(K, generator=g, device=DEV)}
    if case["bias"]:
        d["b"] = 0.1 * torch.randn(K, generator=g, device=DEV)
    if case["train"]:
        d["dy"] = torch.randn(rows, K, generator=g, device=DEV).to(ty)
        if case["res"]:
            d["res"] = torch.randn(rows, K, generator=g, device=DEV).to(tx)
    return d


def _adamw_inputs(case, seed):
    """Flat buffers in which every tensor starts on a whole block; what lies between is zero."""
    g = _gen(seed)
    count, n = case["tensors"], case["n"]
    wide = -(-n // BLOCK) * BLOCK
    total = count * wide

    def flat(make, dtype):
        t = torch.zeros(count, wide, dtype=dtype, device=DEV)
        t[:, :n] = make
        return t.view(-1)

    def normal(scale):
        return torch.randn(count, n, generator=g, device=DEV).mul_(scale)

    d = {"p": flat(normal(0.02), TYPES[case["p"]]), "g": flat(normal(1e-3), TYPES[case["g"]]),
         "decay": [DECAY * (i % 2 == 0) for i in range(count)], "step": 100}
    if case["copy"] != "none":
        d["copy"] = torch.zeros(total, dtype=TYPES[case["copy"]], device=DEV)
    if case["bits"] == 32:
        d["m"] = flat(normal(3e-4), torch.float32)
        d["v"] = flat(normal(1e-3).square_().add_(1e-7), torch.float32)
    else:
        # Codes of a state in the middle of a run: a sign and 7 bits, or 8 bits, of magnitude,
        # more of the larger ones, with the largest binade present in every block.
        def codes(top, sign):
            u = torch.rand(count, n, generator=g, device=DEV).sqrt_().mul_(top + 1)
            c = u.clamp_(max=top).to(torch.uint8)
            c[:, ::BLOCK] = top
            return c | (torch.randint(0, 2, c.shape, generator=g, device=DEV, dtype=torch.uint8) << 7
                        if sign else 0)
        d["m"] = flat(codes(127, True), torch.uint8)
        d["v"] = flat(codes(255, False), torch.uint8)
        # scale bytes: 2^(byte-127), so that the largest values are near 2^-10
        d["ms"] = torch.randint(100, 104, (total // BLOCK,), generator=g, device=DEV).to(torch.uint8)
        d["vs"] = torch.randint(101, 104, (total // BLOCK,), generator=g, device=DEV).to(torch.uint8)
    return d


def _segments(case, seed):
    """Row offsets [segments + 1] and adapter numbers [segments] (-1: none)."""
    r = random.Random(int(seed) * 7 + 1)
    S, T = case["segments"], case["T"]
    cuts = sorted(r.sample(range(1, T), S - 1)) if S > 1 else []
    if T == S:
        cuts = list(range(1, T))
    used = [i % case["adapters"] for i in range(S - case["bare"])]
    if case["adapters"] >= S:
        used = r.sample(range(case["adapters"]), S - case["bare"])
    ids = used + [-1] * case["bare"]
    r.shuffle(ids)
    return [0, *cuts, T], ids


def _ranks(case):
    """Ranks of the adapters: half of them the widest, others narrower or odd."""
    R = case["R"]
    return [(R, R, R // 2, R - 3)[i % 4] for i in range(case["adapters"])]


def _adapter_inputs(case, seed):
    g = _gen(seed)
    T, K, N, R, n = (case[k] for k in ("T", "K", "N", "R", "adapters"))
    tx = TYPES[case["x"]]
    ty = tx if case["y"] == "x" else TYPES[case["y"]]
    off, ids = _segments(case, seed)
    r = random.Random(int(seed) * 5 + 3)
    d = {"x": _acts(g, T, K).to(tx), "off": off, "ids": ids,
         "a": torch.randn(n, R, K, generator=g, device=DEV).mul_(K ** -0.5).to(tx),
         "b": torch.randn(n, N, R, generator=g, device=DEV).mul_(0.05).to(tx),
         "y": torch.randn(T, N, generator=g, device=DEV).to(ty),
         "scales": torch.tensor([2.0 * r.choice((1.0, 0.5, 0.25)) for _ in range(n)], device=DEV),
         "ranks": torch.tensor(_ranks(case), dtype=torch.int32, device=DEV),
         "d_off": torch.tensor(off, dtype=torch.int32, device=DEV),
         "d_ids": torch.tensor(ids, dtype=torch.int32, device=DEV)}
    if case["train"]:
        d["dy"] = torch.randn(T, N, generator=g, device=DEV).to(tx)
        d["dx"] = torch.randn(T, K, generator=g, device=DEV).to(tx)
    return d


_INPUTS = {"norm": _norm_inputs, "adamw": _adamw_inputs, "adapters": _adapter_inputs}


def prepare(case, seed):
    """Inputs and the buffers, plan and state of a program that repeats the call."""
    kind = case["kind"]
    st = {"case": case, **_INPUTS[kind](case, seed)}
    if not own:
        return st
    from paper_2607_14618_gb300 import polyq
    if kind == "norm":
        rows, K = st["x"].shape
        st["out"] = torch.empty(rows, K, dtype=TYPES[case["y"]], device=DEV)
        if case["train"]:
            st["stats"] = polyq.layernorm_stats(rows, DEV)
            st["ws"] = polyq.layernorm_workspace(rows, K, DEV)
            st["dx"] = torch.empty_like(st["x"])
            st["dw"] = torch.empty_like(st["w"])
            st["db"] = torch.empty_like(st["b"]) if case["bias"] else None
    elif kind == "adamw":
        count, n = case["tensors"], case["n"]

        def split(flat):
            return [t[:n] for t in flat.view(count, -1)]

        state = polyq.AdamState([n] * count, case["bits"], DEV)
        state.m.copy_(st["m"])
        state.v.copy_(st["v"])
        if case["bits"] == 8:
            state.m_scales.copy_(st["ms"])
            state.v_scales.copy_(st["vs"])
            st["mv"] = [torch.empty(st["m"].numel(), dtype=torch.bfloat16, device=DEV)
                        for _ in range(2)]
        st["state"] = state
        st["plan"] = polyq.AdamW(split(st["p"]), split(st["g"]), state,
                                 copies=split(st["copy"]) if "copy" in st else None,
                                 weight_decay=st["decay"])
    else:
        n, R, K, N = case["adapters"], case["R"], case["K"], case["N"]
        st["ws"] = polyq.adapters_workspace(case["T"], R, DEV)
        st["out"] = torch.empty_like(st["y"])
        if case["train"]:
            st["saved"] = polyq.adapters_saved(case["T"], R, DEV)
            st["dx_out"] = torch.empty_like(st["dx"])
            st["da"] = torch.empty(n, R, K, dtype=torch.float32, device=DEV)
            st["db"] = torch.empty(n, N, R, dtype=torch.float32, device=DEV)
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_norm(st):
    case = st["case"]
    x, w = st["x"].float(), st["w"]
    mean = x.mean(1, keepdim=True) if case["center"] else 0.0
    c = x - mean
    rstd = 1 / torch.sqrt(c.square().mean(1, keepdim=True) + EPS)
    hat = c * rstd
    y = hat * w
    if case["bias"]:
        y = y + st["b"]
    out = {"y": y.to(TYPES[case["y"]])}
    if case["train"]:
        dy = st["dy"].float()
        g = dy * w
        dx = g - hat * (g * hat).mean(1, keepdim=True)
        if case["center"]:
            dx = dx - g.mean(1, keepdim=True)
        dx = dx * rstd
        if case["res"]:
            dx = dx + st["res"].float()
        out["dx"] = dx.to(st["x"].dtype)
        out["dw"] = (dy * hat).sum(0)
        if case["bias"]:
            out["db"] = dy.sum(0)
    return out


def _mix(h):
    """One round of the state's hash, on 32-bit numbers held in int64."""
    h = (h ^ (h >> 16)) * 0x9E2D58A5 & 0xFFFFFFFF
    return (h ^ (h >> 15)) * 0x6C62272D & 0xFFFFFFFF


def _noise(seed, n):
    """32 random bits for each of n elements: what an 8-bit state is rounded with."""
    block = torch.arange(n // BLOCK, dtype=torch.int64, device=DEV)
    first = _mix(torch.tensor((seed + 1) & 0xFFFFFFFF, device=DEV))
    key = _mix(_mix(block & 0xFFFFFFFF ^ first) ^ (block >> 32) ^ (seed >> 32))
    h = _mix(key[:, None] + torch.arange(BLOCK, device=DEV) * 0x9E3779B1 & 0xFFFFFFFF)
    return h ^ (h >> 16)


def _decode(c, s, mantissa):
    """fp32 values [blocks][256] of codes without a sign: a small IEEE format of `mantissa` bits
    whose smallest normal number is 1, times 2^(s-127)."""
    one = 1 << mantissa
    i = torch.arange(16 * one, device=DEV)
    e, f = i // one, (i % one).double() / one
    grid = torch.where(e > 0, (1 + f) * torch.exp2(e - 1.0), f).float()
    return grid[c.view(-1, BLOCK).int()] * torch.exp2(s.double() - 127).float()[:, None]


def _encode(a, u, mantissa, top):
    """Codes and scale bytes of fp32 magnitudes [blocks][256]: the smallest scale with which the
    largest one is within the codes; rounded up where the 16-bit fraction u and what lies behind
    the last place carry."""
    one = 1 << mantissa
    peak = a.amax(1)
    f, e = torch.frexp(peak)
    s = torch.where(peak > 0, e + 112 + (f > 1 - 0.5 / one), 0).clamp(min=0)
    t = a * torch.exp2(127 - s.double()).float()[:, None]
    f, e = torch.frexp(t)
    part = torch.where(e > 0, f * (2 * one), t * one)
    c = torch.floor(part.double() + u.double() / 65536).int() + (e - 1).clamp(min=0) * one
    return c.clamp(max=top).to(torch.uint8), s.to(torch.uint8)


def _plain_adamw(st):
    case = st["case"]
    st["step"] += 1
    t = st["step"]
    wide = st["p"].numel() // case["tensors"]
    decay = torch.tensor(st["decay"], device=DEV).repeat_interleave(wide)
    p, g = st["p"].float(), st["g"].float()
    eight = case["bits"] == 8
    if eight:
        sign = 1.0 - 2.0 * (st["m"] >> 7).float()
        m = _decode(st["m"] & 127, st["ms"], 3).view(-1) * sign
        v = _decode(st["v"], st["vs"], 4).view(-1).square()
    else:
        m, v = st["m"], st["v"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    root = torch.sqrt(v)
    step = LR / (1 - BETA1 ** t)
    p = p * (1 - LR * decay) - step * m / (root / math.sqrt(1 - BETA2 ** t) + ADAM_EPS)
    st["p"].copy_(p)
    out = {"p": st["p"]}
    if "copy" in st:
        st["copy"].copy_(st["p"])
        out["copy"] = st["copy"]
    if not eight:
        st["m"].copy_(m)
        st["v"].copy_(v)
        return {**out, "m": st["m"], "v": st["v"]}
    u = _noise(t, m.numel())
    root = root.view(-1, BLOCK)
    cm, ms = _encode(m.abs().view(-1, BLOCK), u & 0xFFFF, 3, 127)
    cv, vs = _encode(root, u >> 16, 4, 255)
    cv = torch.maximum(cv, (root > 0).to(torch.uint8))
    st["m"].copy_((cm + ((m < 0).view(-1, BLOCK) & (cm > 0)) * 128).view(-1))
    st["v"].copy_(cv.view(-1))
    st["ms"].copy_(ms)
    st["vs"].copy_(vs)
    mv = _decode(cm, ms, 3).view(-1) * (1 - 2 * (m < 0).float())
    return {**out, "m": mv.to(torch.bfloat16), "v": _decode(cv, vs, 4).view(-1).to(torch.bfloat16)}


def _plain_adapters(st):
    """Adapters next to each other along the rank: a row's product with all of them, of which its
    own is kept; with few rows their own adapters, gathered."""
    case = st["case"]
    T, R, n = case["T"], case["R"], case["adapters"]
    lengths = st["d_off"][1:] - st["d_off"][:-1]
    row = torch.repeat_interleave(st["d_ids"].long(), lengths, output_size=T)
    kept = torch.arange(R, device=DEV) < st["ranks"][:, None]  # [n][R]
    x, y = st["x"].float(), st["y"].float()
    if T <= 64 and not case["train"]:
        mine = row.clamp(min=0)
        keep = (kept[mine] & (row >= 0)[:, None]).float()
        v = (st["a"][mine].float() @ x[:, :, None])[:, :, 0] * keep * st["scales"][mine][:, None]
        return (y + (st["b"][mine].float() @ v[:, :, None])[:, :, 0]).to(st["y"].dtype)
    keep = ((row[:, None] == torch.arange(n, device=DEV))[:, :, None] & kept).float()
    scaled = (keep * st["scales"][:, None]).reshape(T, n * R)
    keep = keep.reshape(T, n * R)
    a = st["a"].float().reshape(n * R, -1)
    b = st["b"].float().permute(0, 2, 1).reshape(n * R, -1)
    v = (x @ a.T) * keep
    y = (y + (v * scaled) @ b).to(st["y"].dtype)
    if not case["train"]:
        return y
    dy = st["dy"].float()
    dv = (dy @ b.T) * scaled
    dx = (st["dx"].float() + dv @ a).to(st["x"].dtype)
    return {"y": y, "dx": dx, "da": (dv.T @ x).view(n, R, -1),
            "db": ((v * scaled).T @ dy).view(n, R, -1).permute(0, 2, 1).contiguous()}


def run(st):
    """One pass through the case's operator."""
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"norm": _plain_norm, "adamw": _plain_adamw, "adapters": _plain_adapters}[kind](st)
    from paper_2607_14618_gb300 import polyq
    if kind == "norm":
        y = polyq.layernorm_forward(st["x"], st["w"], st.get("b"), eps=EPS, center=case["center"],
                                    y=st["out"], stats=st.get("stats"))
        if not case["train"]:
            return {"y": y}
        dx, dw, db = polyq.layernorm_backward(
            st["x"], st["w"], st["stats"], st["dy"], center=case["center"], dx=st["dx"],
            dweight=st["dw"], dbias=st["db"], need_bias=case["bias"], residual=st.get("res"),
            workspace=st["ws"])
        out = {"y": y, "dx": dx, "dw": dw}
        return {**out, "db": db} if case["bias"] else out
    if kind == "adamw":
        st["step"] += 1
        st["plan"].step(LR, st["step"], betas=(BETA1, BETA2), eps=ADAM_EPS, seed=st["step"])
        out = {"p": st["p"], "copy": st["copy"]} if "copy" in st else {"p": st["p"]}
        if case["bits"] == 32:
            return {**out, "m": st["state"].m, "v": st["state"].v}
        m, v = st["state"].values(*st["mv"])
        return {**out, "m": m, "v": v}
    y = polyq.adapters_forward(st["x"], st["a"], st["b"], st["d_off"], st["d_ids"],
                               scales=st["scales"], ranks=st["ranks"], residual=st["y"],
                               y=st["out"], saved=st.get("saved"), workspace=st["ws"])
    if not case["train"]:
        return y
    dx, da, db = polyq.adapters_backward(
        st["x"], st["a"], st["b"], st["saved"], st["dy"], st["d_off"], st["d_ids"],
        scales=st["scales"], ranks=st["ranks"], residual=st["dx"], dx=st["dx_out"], da=st["da"],
        db=st["db"], workspace=st["ws"])
    return {"y": y, "dx": dx, "da": da, "db": db}


# ---------------------------------------------------------------------------
# work and the definition in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    """Inputs in and results out once; two operations a multiplication and addition.  A norm's
    training step reads x, dy and the residual's gradient and writes y and dx.  Adapters read x,
    dy, the projection's result and its input's gradient, and the adapters that requests use, in
    their own ranks, and write the two sums and every adapter's gradient."""
    kind = case["kind"]
    if kind == "norm":
        n, K = case["rows"] * case["K"], case["K"]
        moved = n * (BYTES[case["x"]] + BYTES[case["y"]]) + 4 * K * (1 + case["bias"])
        flops = 6.0 * n
        if case["train"]:
            moved += n * (BYTES[case["y"]] + BYTES[case["x"]] * (1 + case["res"]))
            moved += 4 * K * (1 + case["bias"])
            flops += 12.0 * n
        return {"bytes": moved, "flops": flops}
    if kind == "adamw":
        n = case["tensors"] * case["n"]
        # 8 bits: both codes in and out, the two values out in bf16
        each = 2 * BYTES[case["p"]] + BYTES[case["g"]] + BYTES[case["copy"]]
        each += 16 if case["bits"] == 32 else 8
        return {"bytes": float(n * each), "flops": 16.0 * n}
    T, K, N, R = (case[k] for k in ("T", "K", "N", "R"))
    by = BYTES["bf16"] if case["y"] == "x" else BYTES[case["y"]]
    used = min(case["adapters"], case["segments"] - case["bare"])
    rank = sum(_ranks(case)) / case["adapters"]
    moved = 2 * T * K + 2 * used * rank * (K + N) + 2 * by * T * N
    flops = 2.0 * T * rank * (K + N)
    if case["train"]:
        moved += 2 * T * N + 2 * 2 * T * K + 4 * case["adapters"] * R * (K + N)
        flops *= 3
    return {"bytes": float(moved), "flops": flops}


def _exact_norm(case, d):
    x, w = d["x"].double(), d["w"].double()
    n = x.shape[1]
    if case["center"]:
        x = x - torch.sum(x, 1, True) / n
    var = torch.sum(x * x, 1, True) / n + EPS
    xh = x / torch.sqrt(var)
    out = {"y": torch.addcmul(d["b"].double(), xh, w) if case["bias"] else xh * w}
    if case["train"]:
        dy = d["dy"].double()
        out["dw"] = torch.einsum("rk,rk->k", dy, xh)
        if case["bias"]:
            out["db"] = torch.einsum("rk->k", dy)
        dh = dy * w
        dot = torch.einsum("rk,rk->r", dh, xh)[:, None]
        dx = dh * n - xh * dot
        if case["center"]:
            dx = dx - torch.sum(dh, 1, True)
        dx = dx / (n * torch.sqrt(var))
        out["dx"] = dx + d["res"].double() if case["res"] else dx
    return out


def _exact_bits(seed, count):
    """The 32 bits of `count` elements, in unsigned arithmetic modulo 2^32."""
    M = (1 << 32) - 1

    def scramble(v):
        v = torch.bitwise_and(torch.bitwise_xor(v, v >> 16) * 2653771941, M)
        return torch.bitwise_and(torch.bitwise_xor(v, v >> 15) * 1818371885, M)

    i = torch.arange(count, dtype=torch.int64, device=DEV)
    b, j = i >> 8, i & 255
    start = scramble(torch.tensor([(int(seed) + 1) & M], device=DEV))
    key = scramble(scramble(torch.bitwise_and(b, M) ^ start) ^ (b >> 32) ^ (int(seed) >> 32))
    v = scramble(torch.bitwise_and(key + j * 2654435761, M))
    return v ^ (v >> 16)


def _exact_grid(mantissa, top):
    """The magnitudes of all codes, ascending."""
    vals, step, at = [], 1.0 / (1 << mantissa), 0.0
    for c in range(top + 1):
        vals.append(at)
        if c and c % (1 << mantissa) == 0 and c > (1 << mantissa):
            step *= 2
        at += step
    return torch.tensor(vals, dtype=torch.float64, device=DEV)


def _exact_round(a, frac, mantissa, top):
    """The value of the grid that `a` [blocks][256] is rounded to: the lower neighbour, or the
    upper one where a's fraction of the step and `frac` make at least one."""
    grid = _exact_grid(mantissa, top)
    peak = torch.amax(a, 1, True)
    e = torch.floor(torch.log2(torch.where(peak > 0, peak, torch.full_like(peak, 2.0 ** -126))))
    e = e + (torch.exp2(e + 1) <= peak).double() - (torch.exp2(e) > peak).double()
    e = e + (peak > grid[top] * torch.exp2(e - 14)).double()
    unit = torch.exp2((e - 14).clamp(min=-127))
    t = a / unit
    low = torch.bucketize(t, grid, right=True) - 1
    high = (low + 1).clamp(max=top)
    step = torch.where(low < top, grid[high] - grid[low], grid[top] - grid[top - 1])
    up = (t - grid[low]) / step + frac >= 1
    return grid[torch.where(up, high, low)] * unit, unit, grid


def _exact_adamw(case, d):
    t = d["step"] + 1
    rows = case["tensors"]
    p, g = d["p"].double(), d["g"].double()
    if case["bits"] == 8:
        grid = _exact_grid(3, 127)
        m = grid[(d["m"] & 127).long()] * torch.where(d["m"] > 127, -1.0, 1.0).double()
        m = m * torch.exp2(d["ms"].double() - 127).repeat_interleave(BLOCK)
        v = _exact_grid(4, 255)[d["v"].long()] * torch.exp2(d["vs"].double() - 127).repeat_interleave(BLOCK)
        v = v * v
    else:
        m, v = d["m"].double(), d["v"].double()
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g * g, v, BETA2)
    hat = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
    lam = torch.tensor(d["decay"], dtype=torch.float64, device=DEV)[:, None]
    p = p.view(rows, -1)
    p = (p - LR * lam * p).view(-1) - LR * hat
    out = {"p": p, "copy": p} if "copy" in d else {"p": p}
    if case["bits"] == 32:
        return {**out, "m": m, "v": v}
    u = _exact_bits(t, m.numel())
    sign = torch.sign(m)
    m, _, _ = _exact_round(m.abs().view(-1, BLOCK), (u & 65535).double().view(-1, BLOCK) / 65536, 3, 127)
    root = v.sqrt().view(-1, BLOCK)
    r, unit, grid = _exact_round(root, (u >> 16).double().view(-1, BLOCK) / 65536, 4, 255)
    r = torch.where((r == 0) & (root > 0), unit * grid[1], r)
    return {**out, "m": m.view(-1) * sign, "v": r.view(-1)}


def _exact_adapters(case, d):
    """Segment by segment."""
    x, y, a, b = (d[k].double() for k in ("x", "y", "a", "b"))
    train = case["train"]
    if train:
        dy, dx = d["dy"].double(), d["dx"].double()
        da, db = torch.zeros_like(a), torch.zeros_like(b)
    for i, s, e in zip(d["ids"], d["off"], d["off"][1:]):
        if i < 0:
            continue
        r, c = int(d["ranks"][i]), float(d["scales"][i])
        A, B = a[i, :r], b[i, :, :r]
        v = torch.mm(x[s:e], A.t())
        y[s:e] += c * torch.mm(v, B.t())
        if train:
            dv = c * torch.mm(dy[s:e], B)
            dx[s:e] += torch.mm(dv, A)
            da[i, :r] += torch.mm(dv.t(), x[s:e])
            db[i, :, :r] += c * torch.mm(dy[s:e].t(), v)
    return {"y": y, "dx": dx, "da": da, "db": db} if train else y


def exact(case, seed):
    """The outputs of the case in 64 bits, from the definitions."""
    kind = case["kind"]
    d = _INPUTS[kind](case, seed)
    return {"norm": _exact_norm, "adamw": _exact_adamw, "adapters": _exact_adapters}[kind](case, d)
