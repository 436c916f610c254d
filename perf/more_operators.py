"""Gated layers, group norm with an activation over channels-last maps, and dropout, as a training loop and a service call them: the gated layer's
forward pass (both int8 projections, the activation, the product; what it keeps goes into 8-bit checkpoints) and its gradient from those checkpoints, the
norm forward and backward, from its input or from the checkpoint of the normalised maps, and dropout with a residual, whose mask is the library's random word.

Sizes are those of `workloads` (784-500-500 at 64 samples, 784-2000-2000, 4096-4096 at 8192 samples per set, 32x32 maps of 256 images, 4x4 maps of the last
stage of a residual stack) and others of the same ranges.  int8 matrices have rows of `_pitch` bytes; a checkpoint holds int8 codes and one power-of-two
scale per 32 columns as an exponent byte.

`run` is the plain form in 32 bits, or the library's calls where `own` is true; `exact` restates the definitions in 64 bits."""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
ACTS = {"identity": 0, "relu": 1, "gelu": 2, "silu": 3}
EPS = 1e-5
MOST_VALUES = 16384 * 4096          # of the largest listed matrices and maps
MOST_MACS = 16384 * 4096 * 4096     # of each projection of the largest listed gated layer


def listed():
    return [
        # one sample through a gated layer in service: the weights are read once, latency
        {"name": "gated_forward_token", "op": "gated_forward", "rows": 1, "n": 4096, "k": 4096, "dtype": "bfloat16",
         "act": "silu", "kept": False},
        # the 2000-wide layers of an ordinary batch, both sets: training, rows and columns that end inside tiles
        {"name": "gated_forward_batch", "op": "gated_forward", "rows": 2048, "n": 2000, "k": 2000, "dtype": "float32",
         "act": "gelu", "kept": True},
        # the large dense layers, both sets, training
        {"name": "gated_forward_large", "op": "gated_forward", "rows": 16384, "n": 4096, "k": 4096, "dtype": "bfloat16",
         "act": "silu", "kept": True},
        # a small batch of the MNIST-shaped network: latency, the goodness' own gradient alone
        {"name": "gated_backward_small", "op": "gated_backward", "rows": 128, "n": 500, "dtype": "float32", "act": "gelu",
         "upper": False, "goodness": True},
        # the large dense layers, both sets: the goodness' own gradient and the one from above
        {"name": "gated_backward_large", "op": "gated_backward", "rows": 16384, "n": 4096, "dtype": "bfloat16",
         "act": "silu", "upper": True, "goodness": True},
        # one image in service: latency
        {"name": "group_norm_forward_image", "op": "group_norm_forward", "samples": 1, "side": 32, "channels": 128,
         "groups": 32, "dtype": "bfloat16", "params": "same", "act": "silu", "kept": False, "stochastic": False},
        # 32x32 maps of both sets, training: kept with stochastic rounding
        {"name": "group_norm_forward_maps", "op": "group_norm_forward", "samples": 512, "side": 32, "channels": 128,
         "groups": 32, "dtype": "bfloat16", "params": "float32", "act": "relu", "kept": True, "stochastic": True},
        # a few large images, groups that end inside chunks of eight channels: no workgroup holds a group
        {"name": "group_norm_forward_photos", "op": "group_norm_forward", "samples": 8, "side": 113, "channels": 120,
         "groups": 10, "dtype": "float32", "params": "float32", "act": "gelu", "kept": False, "stochastic": False},
        # the last stage of a residual stack, both sets: short columns, many channels, nothing was checkpointed
        {"name": "group_norm_backward_stage", "op": "group_norm_backward", "samples": 512, "side": 4, "channels": 512,
         "groups": 32, "dtype": "float32", "params": "float32", "act": "silu", "kept": False, "upper": True, "goodness": True},
        # 32x32 maps of both sets, backward from the checkpoint
        {"name": "group_norm_backward_maps", "op": "group_norm_backward", "samples": 512, "side": 32, "channels": 128,
         "groups": 32, "dtype": "bfloat16", "params": "float32", "act": "silu", "kept": True, "upper": True, "goodness": False},
        # activities of a small batch of the MNIST-shaped network: latency
        {"name": "dropout_small", "op": "dropout", "rows": 64, "cols": 500, "dtype": "float32", "p": 0.5, "residual": False},
        # the large dense layers, both sets, added to what goes around the layer
        {"name": "dropout_large", "op": "dropout", "rows": 16384, "cols": 4096, "dtype": "bfloat16", "p": 0.1, "residual": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["gated_forward", "gated_forward", "gated_backward", "group_norm_forward", "group_norm_forward",
                     "group_norm_backward", "group_norm_backward", "dropout"])
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    act = rng.choice(["identity", "relu", "gelu", "silu"])
    if op == "gated_forward":
        n, k = _log_int(rng, 24, 5000), _log_int(rng, 24, 8000)
        if rng.random() < 0.5:
            n, k = (n + 15) // 16 * 16, (k + 15) // 16 * 16
        rows = _log_int(rng, 1, min(65536, MOST_VALUES // max(n, k), MOST_MACS // (n * k)))
        return {"op": op, "rows": rows, "n": n, "k": k, "dtype": dtype, "act": act, "kept": rng.random() < 0.6}
    if op in ("gated_backward", "dropout"):
        cols = _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = (cols + 15) // 16 * 16
        rows = _log_int(rng, 1, min(262144, MOST_VALUES // ((2 if dtype == "float32" else 1) * cols)))
        if op == "dropout":
            return {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "p": round(rng.uniform(0.02, 0.9), 3),
                    "residual": rng.random() < 0.5}
        upper = rng.random() < 0.7
        return {"op": op, "rows": rows, "n": cols, "dtype": dtype, "act": act, "upper": upper,
                "goodness": not upper or rng.random() < 0.5}
    side = _log_int(rng, 1, 128)
    if rng.random() < 0.5:
        per, groups = _log_int(rng, 1, 64), _log_int(rng, 1, 40)
    else:
        per, groups = 1 << rng.randint(0, 7), 1 << rng.randint(0, 5)
    side = max(side, math.ceil(math.sqrt(24 / per)))    # (the gradient of a group of a few values is what cancellation leaves)
    most = MOST_VALUES // (2 if dtype == "float32" else 1) // (side * side * per * groups)
    case = {"op": op, "samples": _log_int(rng, 1, max(1, min(1024, most))), "side": side, "channels": per * groups, "groups": groups,
            "dtype": dtype, "params": rng.choice(["float32", "same"]), "act": act, "kept": rng.random() < 0.5}
    if op == "group_norm_forward":
        return case | {"stochastic": case["kept"] and rng.random() < 0.5}
    if act == "relu" and dtype == "float32":
        case["act"] = "silu"    # one argument rounded across ReLU's border is more than all other roundings of an fp32 gradient
    upper = rng.random() < 0.7
    return case | {"upper": upper, "goodness": not upper or rng.random() < 0.5}


# --- layout ---------------------------------------------------------------------------------------------------------
def _pitch(cols):
    """Bytes between rows of 8-bit matrices: a multiple of 16, of 128 for long rows."""
    return (cols + 127) // 128 * 128 if cols > 512 else (cols + 15) // 16 * 16


def _blocks(cols):
    return (cols + BLOCK - 1) // BLOCK


def _activities(g, rows, cols, of_row):
    """Activities: columns of different widths and offsets, a few of them far wider, samples of different sizes (of_row: rows of one)."""
    wide = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    wide = torch.where(torch.rand(cols, device="cuda", generator=g) < 0.005, wide * 12, wide)
    offset = 0.3 * torch.randn(cols, device="cuda", generator=g)
    size = torch.exp(0.4 * torch.randn(rows // of_row, 1, device="cuda", generator=g)).repeat_interleave(of_row, 0)
    return torch.randn(rows, cols, device="cuda", generator=g).mul_(wide).add_(offset).mul_(size)


def _gradients(g, rows, cols, of_row):
    """A gradient: samples of different sizes (their loss derivatives), columns with a direction of their own."""
    size = (0.02 * torch.exp(0.7 * torch.randn(rows // of_row, 1, device="cuda", generator=g))).repeat_interleave(of_row, 0)
    return torch.randn(rows, cols, device="cuda", generator=g).add_(0.1 * torch.randn(cols, device="cuda", generator=g)).mul_(size)


def _quantised(x):
    """Per-tensor int8 codes with their row pitch, and the scale, as the library's quantiser leaves them (rounded to nearest)."""
    scale = x.abs().amax() / 127
    q = torch.zeros(x.shape[0], _pitch(x.shape[1]), dtype=torch.int8, device="cuda")
    q[:, : x.shape[1]] = torch.round(x / scale).clamp_(-127, 127)
    return q, scale.reshape(1)


def prepare(case, seed):
    g, dtype, op = torch.Generator(device="cuda").manual_seed(seed), TYPES[case["dtype"]], case["op"]
    s = {"case": case, "sr_seed": seed * 7919 + 11, "tag": (seed % 1000 + 1) << 20}
    empty = lambda *shape, of=torch.float32: torch.empty(shape, dtype=of, device="cuda")  # noqa: E731
    checkpoint = lambda rows, cols: (empty(rows, _pitch(cols), of=torch.int8), empty(rows, _pitch(_blocks(cols)), of=torch.uint8))  # noqa: E731
    if op == "gated_forward":
        rows, n, k = case["rows"], case["n"], case["k"]
        s["a_q"], s["s_a"] = _quantised(torch.randn(rows, k, device="cuda", generator=g).mul_(torch.exp(0.3 * torch.randn(k, device="cuda", generator=g))))
        # projections of about unit size
        s["w_q"], s["s_w"] = _quantised((torch.rand(2 * n, k, device="cuda", generator=g) * 2 - 1) * math.sqrt(2.5 / k))
        s |= {"y": empty(rows, n, of=dtype), "goodness": empty(rows), "g": (None, None), "u": (None, None)}
        if case["kept"]:
            s |= {"g": checkpoint(rows, n), "u": checkpoint(rows, n), "back_g": empty(rows, n, of=torch.bfloat16), "back_u": empty(rows, n, of=torch.bfloat16)}
        return s
    if op == "gated_backward":
        rows, n = case["rows"], case["n"]
        s["g"], s["u"] = (_store(_activities(g, rows, n, 1), None) for _ in range(2))
        s["dy"] = _gradients(g, rows, n, 1).to(dtype) if case["upper"] else None
        s["coeff"] = 0.05 * torch.randn(rows, device="cuda", generator=g) if case["goodness"] else None
        s["d"] = empty(rows, 2 * n, of=dtype)
        return s
    if op == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _activities(g, rows, cols, 1).to(dtype)
        s["r"] = _activities(g, rows, cols, 1).to(dtype) if case["residual"] else None
        s["y"] = empty(rows, cols, of=dtype)
        return s
    samples, pixels, channels, groups = case["samples"], case["side"] ** 2, case["channels"], case["groups"]
    rows = samples * pixels
    of = dtype if case["params"] == "same" else torch.float32
    s["weight"] = (1 + 0.2 * torch.randn(channels, device="cuda", generator=g)).to(of)
    s["bias"] = (0.2 * torch.randn(channels, device="cuda", generator=g)).to(of)
    x = _activities(g, rows, channels, pixels).to(dtype)
    if op == "group_norm_forward":
        s |= {"x": x, "y": empty(rows, channels, of=dtype), "mean": empty(samples, groups), "rstd": empty(samples, groups),
              "goodness": empty(samples), "q": None, "e": None}
        if case["kept"]:
            s["q"], s["e"] = checkpoint(rows, channels)
            s["back"] = empty(rows, channels, of=torch.bfloat16)
        return s
    grouped = x.float().view(samples, pixels, groups, -1)
    var, mean = torch.var_mean(grouped, (1, 3), unbiased=False)
    s |= {"mean": mean, "rstd": 1 / torch.sqrt(var + EPS), "x": x, "q": None, "e": None}
    if case["kept"]:
        s["q"], s["e"] = _store(((grouped - mean[:, None, :, None]) * s["rstd"][:, None, :, None]).view(rows, channels), None)
        s["x"] = s["mean"] = None
    s["dy"] = _gradients(g, rows, channels, pixels).to(dtype) if case["upper"] else None
    s["coeff"] = 0.05 * torch.randn(samples, device="cuda", generator=g) if case["goodness"] else None
    return s | {"dx": empty(rows, channels, of=dtype), "dw": empty(channels), "db": empty(channels)}


# --- the plain form: 32 bits, rounded once at the end -----------------------------------------------------------------
def _uniform(rows, cols, seed, tag):
    """The library's random words as uniforms: a 64-bit finaliser of (seed, tag), then a 32-bit mixer per element."""
    m64, m32 = (1 << 64) - 1, 0xFFFFFFFF
    z = (seed + 0x9E3779B97F4A7C15 * (tag + 1)) & m64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m64
    z ^= z >> 31
    v = torch.arange(rows * cols, device="cuda") ^ (z & m32)   # (fewer than 2^32 elements: the high word of the index is 0)
    v = v ^ (v >> 16)
    v = (v * 0x7FEB352D) & m32
    v = v ^ (v >> 15)
    v = (v * 0x846CA68B) & m32
    v = v ^ (v >> 16)
    return (v >> 8).to(torch.float32).reshape(rows, cols) * 2.0**-24


def _store(x, u):
    """Codes and exponent bytes of the fp32 tensor x; u: uniforms for stochastic rounding, or None for nearest-even."""
    rows, cols = x.shape
    nb = _blocks(cols)
    xb = torch.nn.functional.pad(x, (0, nb * BLOCK - cols)).reshape(rows, nb, BLOCK)
    amax = xb.abs().amax(2)
    frac, exp = torch.frexp(amax)                       # amax = frac * 2^exp, frac in [1/2, 1)
    s = torch.where(frac <= 127 / 128, exp - 7, exp - 6).clamp(max=121)
    some = amax >= 2.0**-100
    s = torch.where(some, s, torch.zeros_like(s))
    t = xb * torch.where(some, torch.ldexp(torch.ones_like(amax), -s), torch.zeros_like(amax))[..., None]
    t = t.reshape(rows, nb * BLOCK)[:, :cols]
    if u is None:
        code = torch.round(t)
    else:
        low = torch.floor(t)
        code = low + (u < t - low)
    q = torch.zeros(rows, _pitch(cols), dtype=torch.int8, device="cuda")
    q[:, :cols] = code.clamp(-127, 127)
    e = torch.zeros(rows, _pitch(nb), dtype=torch.uint8, device="cuda")
    e[:, :nb] = s + 127
    return q, e


def _load(q, e, cols):
    s = torch.exp2(e[:, :_blocks(cols)].float() - 127)
    return q[:, :cols].float() * s.repeat_interleave(BLOCK, 1)[:, :cols]


def _act(kind, u):
    """An activation and its derivative."""
    if kind == "relu":
        return u.clamp(min=0), (u > 0).float()
    if kind == "gelu":
        phi = 0.5 * (1 + torch.erf(u * math.sqrt(0.5)))
        return u * phi, phi + u * torch.exp(-0.5 * u * u) * (1 / math.sqrt(2 * math.pi))
    if kind == "silu":
        sig = 1 / (1 + torch.exp(-u))
        return u * sig, sig * (1 + u * (1 - sig))
    return u, torch.ones_like(u)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "gated_forward":
        n, k = case["n"], case["k"]
        # (sums of these sizes are whole numbers of fewer than 25 bits: exact in 32 bits, in any order)
        t = (s["a_q"][:, :k].float() @ s["w_q"][:, :k].float().t()) * (s["s_a"] * s["s_w"])
        g, u = t[:, :n], t[:, n:]
        y = _act(case["act"], g)[0] * u
        out = {"y": y.to(TYPES[case["dtype"]]), "goodness": (y * y).sum(1)}
        if case["kept"]:
            out["kept_g"], out["kept_u"] = (_load(*_store(v, None), n).to(torch.bfloat16) for v in (g, u))
        return out
    if op == "gated_backward":
        n = case["n"]
        g, u = _load(*s["g"], n), _load(*s["u"], n)
        f, d = _act(case["act"], g)
        t = s["dy"].float() if case["upper"] else torch.zeros_like(g)
        if case["goodness"]:
            t = t + 2 * s["coeff"][:, None] * (f * u)
        return {"d": torch.cat([t * u * d, t * f], 1).to(TYPES[case["dtype"]])}
    if op == "dropout":
        keep = _uniform(case["rows"], case["cols"], s["sr_seed"], s["tag"]) >= case["p"]
        y = torch.where(keep, s["x"].float() * (1 / (1 - case["p"])), 0.0)
        if case["residual"]:
            y = y + s["r"].float()
        return {"y": y.to(s["x"].dtype)}
    samples, pixels, channels, groups = case["samples"], case["side"] ** 2, case["channels"], case["groups"]
    rows, m = samples * pixels, pixels * (channels // groups)
    weight, bias = s["weight"].float(), s["bias"].float()
    if op == "group_norm_forward":
        x = s["x"].float().view(samples, pixels, groups, -1)
        mean = x.mean((1, 3))
        dev = x - mean[:, None, :, None]
        rstd = 1 / torch.sqrt((dev * dev).mean((1, 3)) + EPS)
        h = (dev * rstd[:, None, :, None]).view(rows, channels)
        y = _act(case["act"], h * weight + bias)[0]
        out = {"y": y.to(s["x"].dtype), "mean": mean, "rstd": rstd, "goodness": (y * y).view(samples, -1).sum(1)}
        if case["kept"]:
            u = _uniform(rows, channels, s["sr_seed"], s["tag"]) if case["stochastic"] else None
            out["kept"] = _load(*_store(h, u), channels).to(torch.bfloat16)
        return out
    if case["kept"]:
        h = _load(s["q"], s["e"], channels)
    else:
        h = ((s["x"].float().view(samples, pixels, groups, -1) - s["mean"][:, None, :, None]) * s["rstd"][:, None, :, None]).view(rows, channels)
    if case["act"] == "relu":   # the argument's sign, next to the border
        z = (h.double() * weight.double() + bias.double()).float()
    else:
        z = h * weight + bias
    f, d = _act(case["act"], z)
    dz = s["dy"].float() if case["upper"] else torch.zeros_like(z)
    if case["goodness"]:
        dz = dz + 2 * s["coeff"].repeat_interleave(pixels)[:, None] * f
    dz = dz * d
    of_group = lambda v: v.view(samples, pixels, groups, -1).sum((1, 3), keepdim=True) / m  # noqa: E731
    gh = (dz * weight)
    dx = (gh.view(samples, pixels, groups, -1) - of_group(gh) - h.view(samples, pixels, groups, -1) * of_group(gh * h)) * s["rstd"][:, None, :, None]
    return {"dx": dx.reshape(rows, channels).to(TYPES[case["dtype"]]), "dweight": (dz * h).sum(0), "dbias": dz.sum(0)}


# --- the library's calls ------------------------------------------------------------------------------------------------
def _workspace(s, size, *sizes):
    """Kept by the program between its steps."""
    if "ws" not in s:
        s["ws"] = torch.empty(size(*sizes), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _library(s):
    import paper_2506_22771_amd as ff
    case, op = s["case"], s["case"]["op"]
    if op == "gated_forward":
        ws = _workspace(s, ff.ff_gated_workspace_bytes, case["rows"], case["n"], case["k"])
        ff.ff_gated_forward(s["a_q"], s["w_q"], s["s_a"], s["s_w"], case["k"], ACTS[case["act"]], s["y"], s["goodness"], *s["g"], *s["u"], ws)
        out = {"y": s["y"], "goodness": s["goodness"]}
        if case["kept"]:
            ff.ff_ckpt_load(*s["g"], s["back_g"])
            ff.ff_ckpt_load(*s["u"], s["back_u"])
            out |= {"kept_g": s["back_g"], "kept_u": s["back_u"]}
        return out
    if op == "gated_backward":
        n = case["n"]
        ff.ff_gated_backward(*s["g"], *s["u"], ACTS[case["act"]], s["coeff"], s["dy"], s["d"][:, :n], s["d"][:, n:])
        return {"d": s["d"]}
    if op == "dropout":
        ff.ff_dropout(s["x"], s["r"], case["p"], s["sr_seed"], s["tag"], None, s["y"])
        return {"y": s["y"]}
    samples, groups = case["samples"], case["groups"]
    ws = _workspace(s, ff.ff_group_norm_workspace_bytes, samples, case["side"] ** 2, case["channels"], groups)
    if op == "group_norm_forward":
        ff.ff_group_norm_forward(s["x"], samples, groups, s["weight"], s["bias"], EPS, ACTS[case["act"]], s["y"], s["mean"], s["rstd"], s["goodness"],
                                 s["q"], s["e"], ff.ROUND_STOCHASTIC if case["stochastic"] else ff.ROUND_NEAREST, s["sr_seed"], s["tag"], ws)
        out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"], "goodness": s["goodness"]}
        if case["kept"]:
            ff.ff_ckpt_load(s["q"], s["e"], s["back"])
            out["kept"] = s["back"]
        return out
    ff.ff_group_norm_backward(s["dy"], s["coeff"], s["x"], s["mean"], s["q"], s["e"], s["rstd"], samples, groups, s["weight"], s["bias"],
                              ACTS[case["act"]], s["dx"], s["dw"], s["db"], False, ws)
    return {"dx": s["dx"], "dweight": s["dw"], "dbias": s["db"]}


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    size, op = TYPES[case["dtype"]].itemsize, case["op"]
    codes = lambda rows, cols: rows * (cols + _blocks(cols))  # noqa: E731
    if op == "gated_forward":
        rows, n, k = case["rows"], case["n"], case["k"]
        kept = 2 * (2 * codes(rows, n) + 2 * rows * n) if case["kept"] else 0      # written, and read back as bf16 values
        return {"bytes": rows * k + 2 * n * k + rows * n * size + 4 * rows + kept, "flops": 4 * rows * n * k}
    if op == "gated_backward":
        rows, n = case["rows"], case["n"]
        return {"bytes": 2 * codes(rows, n) + rows * n * size * (2 + case["upper"]) + 4 * rows * case["goodness"], "flops": 20 * rows * n}
    if op == "dropout":
        values = case["rows"] * case["cols"]
        return {"bytes": values * size * (2 + case["residual"]), "flops": 3 * values}
    rows, channels, stats = case["samples"] * case["side"] ** 2, case["channels"], case["samples"] * case["groups"]
    values, params = rows * channels, channels * (4 if case["params"] == "float32" else size)
    if op == "group_norm_forward":
        kept = 2 * codes(rows, channels) + 2 * values if case["kept"] else 0
        return {"bytes": 2 * values * size + 2 * params + 8 * stats + 4 * case["samples"] + kept, "flops": 16 * values}
    h = codes(rows, channels) if case["kept"] else values * size + 4 * stats
    return {"bytes": values * size * (1 + case["upper"]) + h + 4 * stats + 2 * params + 8 * channels + 4 * case["samples"] * case["goodness"],
            "flops": 30 * values}


# --- in 64 bits ---------------------------------------------------------------------------------------------------------
def _values64(q, e, cols):
    at = torch.arange(cols, device="cuda")
    return q[:, at].double() * torch.pow(2.0, e.double() - 127)[:, at // BLOCK]


def _kept64(x, u):
    """The values that a checkpoint of x stands for."""
    rows, cols = x.shape
    nb, whole = _blocks(cols), cols // BLOCK
    most = torch.zeros(rows, nb, dtype=torch.float64, device="cuda")
    if whole:
        most[:, :whole] = x[:, : whole * BLOCK].abs().reshape(rows, whole, BLOCK).amax(2)
    if whole < nb:
        most[:, whole] = x[:, whole * BLOCK:].abs().amax(1)
    none = most < 2.0**-100
    s = torch.ceil(torch.log2(torch.where(none, 127.0, most) / 127.0))
    s = torch.where(127.0 * torch.exp2(s) < most, s + 1, s)            # the logarithm's own rounding
    s = torch.where(127.0 * torch.exp2(s - 1) >= most, s - 1, s)
    step = torch.exp2(torch.where(none, 0.0, s.clamp(max=121))).repeat_interleave(BLOCK, 1)[:, :cols]
    t = x / step
    t = torch.round(t) if u is None else torch.floor(t) + (u.double() < t - torch.floor(t)).double()
    return torch.where(none.repeat_interleave(BLOCK, 1)[:, :cols], 0.0, t.clamp(-127, 127)) * step


def _act64(act, u):
    if act == "relu":
        return torch.relu(u), (u > 0).double()
    if act == "gelu":
        low = 0.5 * torch.erfc(-u / math.sqrt(2))
        return u * low, low + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        return u * torch.sigmoid(u), torch.sigmoid(u) + u * torch.sigmoid(u) * torch.sigmoid(-u)
    return u, torch.ones_like(u)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "gated_forward":
        n, k = case["n"], case["k"]
        scale = s["s_a"].double() * s["s_w"].double()
        g = torch.mm(s["a_q"][:, :k].double(), s["w_q"][:n, :k].double().t()) * scale
        u = torch.mm(s["a_q"][:, :k].double(), s["w_q"][n:, :k].double().t()) * scale
        y = _act64(case["act"], g)[0] * u
        out = {"y": y, "goodness": torch.linalg.vecdot(y, y)}
        return out | ({"kept_g": _kept64(g, None), "kept_u": _kept64(u, None)} if case["kept"] else {})
    if op == "gated_backward":
        g, u = _values64(*s["g"], case["n"]), _values64(*s["u"], case["n"])
        f, d = _act64(case["act"], g)
        t = 2 * s["coeff"].double()[:, None] * u * f if case["goodness"] else 0.0
        t = t + (s["dy"].double() if case["upper"] else 0.0)
        return {"d": torch.cat((u * d * t, f * t), 1)}
    if op == "dropout":
        dropped = _uniform(case["rows"], case["cols"], s["sr_seed"], s["tag"]).double() < torch.tensor(case["p"], dtype=torch.float32).double().item()
        y = (s["x"].double() / (1 - case["p"])).masked_fill(dropped, 0)
        return {"y": y + s["r"].double() if case["residual"] else y}
    samples, groups, channels = case["samples"], case["groups"], case["channels"]
    per = channels // groups
    spread = lambda v: v.double().repeat_interleave(per, 1).repeat_interleave(case["side"] ** 2, 0)  # noqa: E731
    weight, bias = s["weight"].double(), s["bias"].double()
    if op == "group_norm_forward":
        x = s["x"].double().reshape(samples, -1, groups, per).transpose(1, 2).reshape(samples, groups, -1)
        var, mean = torch.var_mean(x, 2, unbiased=False)
        rstd = torch.rsqrt(var + EPS)
        h = spread(rstd) * (s["x"].double() - spread(mean))
        y = _act64(case["act"], bias + weight * h)[0]
        out = {"y": y, "mean": mean, "rstd": rstd, "goodness": y.reshape(samples, -1).square().sum(1)}
        if case["kept"]:
            u = _uniform(*h.shape, s["sr_seed"], s["tag"]) if case["stochastic"] else None
            out["kept"] = _kept64(h, u)
        return out
    r = spread(s["rstd"])
    h = _values64(s["q"], s["e"], channels) if case["kept"] else r * (s["x"].double() - spread(s["mean"]))
    f, d = _act64(case["act"], bias + weight * h)
    up = 2 * f * s["coeff"].double().repeat_interleave(case["side"] ** 2)[:, None] if case["goodness"] else 0.0
    dz = d * (up + (s["dy"].double() if case["upper"] else 0.0))
    m = case["side"] ** 2 * per
    sums = lambda v: v.reshape(samples, -1, groups, per).sum(3).sum(1)  # noqa: E731
    dx = r / m * (m * weight * dz - spread(sums(weight * dz)) - h * spread(sums(weight * dz * h)))
    return {"dx": dx, "dweight": torch.linalg.vecdot(dz, h, dim=0), "dbias": dz.sum(0)}
