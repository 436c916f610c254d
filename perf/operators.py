"""Layer norm and 8-bit activation checkpoints as a training loop calls them: the norm forward (what it keeps for the backward pass
goes straight into a checkpoint) and backward, checkpoints of other tensors written and read, the gradient through an activation whose
argument was checkpointed, and the weight gradient of the layer behind a norm, formed from the norm's checkpoint.

Sizes are those of `workloads` (784-500-500 at 64 samples, 784-2000-2000, 4096-4096 at 8192 samples per set, 32x32 maps of 256 images
with 64 to 256 channels) and odd ones of the same ranges.  A checkpoint holds int8 codes, [rows, pitch], and one power-of-two scale
per 32 columns as an exponent byte, [rows, pitch of the blocks].

`run` is the plain form in 32 bits, or the library's calls where `own` is true; `exact` restates the definitions in 64 bits."""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
ACTS = {"identity": 0, "relu": 1, "gelu": 2, "silu": 3}
EPS = 1e-5
MOST_BYTES = 2 * 16384 * 4096       # of the largest listed tensors
MOST_MACS = 16384 * 4096 * 4096     # of the largest listed weight gradient


def listed():
    return [
        # one sample through a network in service: latency
        {"name": "norm_forward_token", "op": "norm_forward", "rows": 1, "cols": 4096, "dtype": "bfloat16",
         "params": "same", "kept": False, "stochastic": False},
        # inputs of the 2000-wide layers of an ordinary batch, both sets: fp32, rows that end inside a block
        {"name": "norm_forward_batch", "op": "norm_forward", "rows": 2048, "cols": 2000, "dtype": "float32",
         "params": "float32", "kept": True, "stochastic": False},
        # inputs of the large dense layers, both sets, checkpointed with stochastic rounding
        {"name": "norm_forward_large", "op": "norm_forward", "rows": 16384, "cols": 4096, "dtype": "bfloat16",
         "params": "float32", "kept": True, "stochastic": True},
        # a norm over the channels of 32x32 maps: many short rows, long columns to sum; nothing was checkpointed
        {"name": "norm_backward_pixels", "op": "norm_backward", "rows": 262144, "cols": 128, "dtype": "float16",
         "params": "float32", "kept": False},
        # the large dense layers, backward from the checkpoint
        {"name": "norm_backward_large", "op": "norm_backward", "rows": 16384, "cols": 4096, "dtype": "bfloat16",
         "params": "same", "kept": True},
        # activities of a small batch of the MNIST-shaped network: latency of the two calls
        {"name": "checkpoint_small", "op": "checkpoint", "rows": 64, "cols": 500, "dtype": "float32", "stochastic": True},
        # activities of the large dense layers, both sets
        {"name": "checkpoint_large", "op": "checkpoint", "rows": 16384, "cols": 4096, "dtype": "bfloat16",
         "stochastic": False},
        # a gradient from the layer above through an activation, odd sizes
        {"name": "act_backward_odd", "op": "act_backward", "rows": 1001, "cols": 870, "dtype": "float16", "act": "silu",
         "goodness": False},
        # the large dense layers: the goodness' own gradient and the one from above
        {"name": "act_backward_large", "op": "act_backward", "rows": 16384, "cols": 4096, "dtype": "bfloat16",
         "act": "gelu", "goodness": True},
        # a small batch of the MNIST-shaped network, both sets
        {"name": "weight_grad_small", "op": "weight_grad", "rows": 128, "n": 500, "k": 784, "dtype": "float32",
         "affine": True},
        # the 2000-wide layers, both sets, fp32 gradients
        {"name": "weight_grad_batch", "op": "weight_grad", "rows": 2048, "n": 2000, "k": 2000, "dtype": "float32",
         "affine": True},
        # the large dense layers, both sets
        {"name": "weight_grad_large", "op": "weight_grad", "rows": 16384, "n": 4096, "k": 4096, "dtype": "bfloat16",
         "affine": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["norm_forward", "norm_forward", "norm_backward", "norm_backward", "checkpoint", "act_backward",
                     "weight_grad", "weight_grad"])
    dtype = rng.choice(["float32", "bfloat16", "float16"])
    if op == "weight_grad":
        n, k = _log_int(rng, 24, 6000), _log_int(rng, 24, 6000)
        if rng.random() < 0.5:
            n, k = (n + 15) // 16 * 16, (k + 15) // 16 * 16
        rows = _log_int(rng, 1, min(262144, MOST_BYTES // (TYPES[dtype].itemsize * max(n, k)), MOST_MACS // (n * k)))
        return {"op": op, "rows": rows, "n": n, "k": k, "dtype": dtype, "affine": rng.random() < 0.7}
    cols = _log_int(rng, 16, 16384)
    if rng.random() < 0.5:
        cols = (cols + 15) // 16 * 16
    case = {"op": op, "rows": _log_int(rng, 1, min(262144, MOST_BYTES // (TYPES[dtype].itemsize * cols))), "cols": cols,
            "dtype": dtype}
    if op in ("norm_forward", "norm_backward"):
        case |= {"params": rng.choice(["float32", "same"]), "kept": rng.random() < 0.6}
    if op in ("norm_forward", "checkpoint"):
        case |= {"stochastic": rng.random() < 0.4 and (op == "checkpoint" or case["kept"])}
    if op == "act_backward":
        case |= {"act": rng.choice(["identity", "relu", "gelu", "silu"]), "goodness": rng.random() < 0.5}
    return case


# --- layout ---------------------------------------------------------------------------------------------------------
def _pitch(cols):
    """Bytes between rows of 8-bit matrices: a multiple of 16, of 128 for long rows."""
    return (cols + 127) // 128 * 128 if cols > 512 else (cols + 15) // 16 * 16


def _blocks(cols):
    return (cols + BLOCK - 1) // BLOCK


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activities(g, rows, cols):
    """A layer's input: columns of different widths and offsets, a few of them far wider, rows of different lengths."""
    wide = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=g))
    wide = torch.where(torch.rand(cols, device="cuda", generator=g) < 0.005, wide * 12, wide)
    offset = 0.3 * torch.randn(cols, device="cuda", generator=g)
    length = torch.exp(0.4 * torch.randn(rows, 1, device="cuda", generator=g))
    return (torch.randn(rows, cols, device="cuda", generator=g) * wide + offset) * length


def _gradients(g, rows, cols):
    """A gradient: rows of different sizes (the samples' loss derivatives), columns with a direction of their own."""
    size = 0.02 * torch.exp(0.7 * torch.randn(rows, 1, device="cuda", generator=g))
    return (torch.randn(rows, cols, device="cuda", generator=g) + 0.1 * torch.randn(cols, device="cuda", generator=g)) * size


def prepare(case, seed):
    g, dtype, op = _generator(seed), TYPES[case["dtype"]], case["op"]
    rows = case["rows"]
    s = {"case": case, "sr_seed": seed * 7919 + 11, "tag": 1 << 20}
    empty = lambda *shape, of=torch.float32: torch.empty(shape, dtype=of, device="cuda")  # noqa: E731
    if op == "weight_grad":
        n, k = case["n"], case["k"]
        s["dy"] = _gradients(g, rows, n).to(dtype)
        x = _activities(g, rows, k)
        x = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, keepdim=True, unbiased=False) + EPS)
        s["q"], s["e"] = _store(x, None)
        s["weight"] = s["bias"] = None
        if case["affine"]:
            s["weight"] = 1 + 0.2 * torch.randn(k, device="cuda", generator=g)
            s["bias"] = 0.2 * torch.randn(k, device="cuda", generator=g)
        s["dw"], s["db"] = empty(n, k), empty(n)
        return s
    cols = case["cols"]
    x = _activities(g, rows, cols).to(dtype)
    if op in ("norm_forward", "norm_backward"):
        of = dtype if case["params"] == "same" else torch.float32
        s["weight"] = (1 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(of)
        s["bias"] = (0.2 * torch.randn(cols, device="cuda", generator=g)).to(of)
    if op == "norm_forward":
        s |= {"x": x, "y": empty(rows, cols, of=dtype), "mean": empty(rows), "rstd": empty(rows), "q": None, "e": None}
        if case["kept"]:
            s["q"], s["e"] = empty(rows, _pitch(cols), of=torch.int8), empty(rows, _pitch(_blocks(cols)), of=torch.uint8)
            s["back"] = empty(rows, cols, of=torch.bfloat16)
    elif op == "norm_backward":
        xf = x.float()
        s["mean"] = xf.mean(1)
        s["rstd"] = 1 / torch.sqrt(xf.var(1, unbiased=False) + EPS)
        if case["kept"]:
            s["q"], s["e"] = _store((xf - s["mean"][:, None]) * s["rstd"][:, None], None)
            s["x"] = s["mean"] = None
        else:
            s |= {"x": x, "q": None, "e": None}
        s["dy"] = _gradients(g, rows, cols).to(dtype)
        s |= {"dx": empty(rows, cols, of=dtype), "dw": empty(cols), "db": empty(cols)}
    elif op == "checkpoint":
        s |= {"x": x, "back": empty(rows, cols, of=dtype)}
        s["q"], s["e"] = empty(rows, _pitch(cols), of=torch.int8), empty(rows, _pitch(_blocks(cols)), of=torch.uint8)
    else:
        s["q"], s["e"] = _store(x.float(), None)
        s["coeff"] = 0.05 * torch.randn(rows, device="cuda", generator=g) if case["goodness"] else None
        s["dy"] = _gradients(g, rows, cols).to(dtype)
        s["dx"] = empty(rows, cols, of=dtype)
    return s


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
    rows = case["rows"]
    if op == "norm_forward":
        x = s["x"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1 / torch.sqrt((d * d).mean(1) + EPS)
        xh = d * rstd[:, None]
        out = {"y": (xh * s["weight"].float() + s["bias"].float()).to(s["x"].dtype), "mean": mean, "rstd": rstd}
        if case["kept"]:
            u = _uniform(rows, case["cols"], s["sr_seed"], s["tag"]) if case["stochastic"] else None
            out["kept"] = _load(*_store(xh, u), case["cols"]).to(torch.bfloat16)
        return out
    if op == "norm_backward":
        dy = s["dy"].float()
        xh = _load(s["q"], s["e"], case["cols"]) if case["kept"] else (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        g = dy * s["weight"].float()
        dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
        return {"dx": dx.to(s["dy"].dtype), "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)}
    if op == "checkpoint":
        u = _uniform(rows, case["cols"], s["sr_seed"], s["tag"]) if case["stochastic"] else None
        q, e = _store(s["x"].float(), u)
        return {"back": _typed(_load(q, e, case["cols"]), s["x"].dtype), "scale": e[:, :_blocks(case["cols"])]}
    if op == "act_backward":
        a, d = _act(case["act"], _load(s["q"], s["e"], case["cols"]))
        dy = s["dy"].float()
        if case["goodness"]:
            dy = dy + 2 * s["coeff"][:, None] * a
        return {"dx": (dy * d).to(s["dy"].dtype)}
    dy = s["dy"].float()
    db = dy.sum(0)
    dw = dy.t() @ _load(s["q"], s["e"], case["k"])
    if case["affine"]:
        dw = dw * s["weight"] + db[:, None] * s["bias"]
    return {"dweight": dw, "dbias": db}


def _typed(x, dtype):
    """Rounded to a type; what lies beyond the range of 16-bit floats (a code rounded up) is their largest value."""
    most = torch.finfo(dtype).max
    return x.clamp(-most, most).to(dtype)


# --- the library's calls ------------------------------------------------------------------------------------------------
def _library(s):
    import paper_2506_22771_amd as ff
    case, op = s["case"], s["case"]["op"]
    if op == "norm_forward":
        ff.ff_layer_norm_forward(s["x"], s["weight"], s["bias"], EPS, s["y"], s["mean"], s["rstd"], s["q"], s["e"],
                                 ff.ROUND_STOCHASTIC if case["stochastic"] else ff.ROUND_NEAREST, s["sr_seed"], s["tag"])
        out = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
        if case["kept"]:
            ff.ff_ckpt_load(s["q"], s["e"], s["back"])
            out["kept"] = s["back"]
        return out
    if op == "norm_backward":
        if "ws" not in s:   # kept by the program between its steps
            s["ws"] = torch.empty(ff.ff_layer_norm_workspace_bytes(case["rows"], case["cols"]), dtype=torch.uint8, device="cuda")
        ff.ff_layer_norm_backward(s["dy"], s["x"], s["mean"], s["q"], s["e"], s["rstd"], s["weight"], s["dx"], s["dw"],
                                  s["db"], False, s["ws"])
        return {"dx": s["dx"], "dweight": s["dw"], "dbias": s["db"]}
    if op == "checkpoint":
        ff.ff_ckpt_store(s["x"], ff.ROUND_STOCHASTIC if case["stochastic"] else ff.ROUND_NEAREST, s["sr_seed"], s["tag"],
                         s["q"], s["e"])
        ff.ff_ckpt_load(s["q"], s["e"], s["back"])
        return {"back": s["back"], "scale": s["e"][:, :_blocks(case["cols"])]}
    if op == "act_backward":
        ff.ff_ckpt_act_backward(s["q"], s["e"], ACTS[case["act"]], s["coeff"], s["dy"], s["dx"])
        return {"dx": s["dx"]}
    if "ws" not in s:
        s["ws"] = torch.empty(ff.ff_ckpt_weight_grad_workspace_bytes(case["rows"], case["n"], case["k"]), dtype=torch.uint8,
                              device="cuda")
    ff.ff_ckpt_weight_grad(s["dy"], s["q"], s["e"], s["weight"], s["bias"], s["dw"], s["db"], False, s["ws"])
    return {"dweight": s["dw"], "dbias": s["db"]}


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    rows, size = case["rows"], TYPES[case["dtype"]].itemsize
    if case["op"] == "weight_grad":
        n, k = case["n"], case["k"]
        kept = rows * (k + _blocks(k))
        return {"bytes": rows * n * size + kept + 4 * n * k + 4 * n + (8 * k if case["affine"] else 0), "flops": 2 * rows * n * k}
    cols = case["cols"]
    values, kept = rows * cols, rows * (cols + _blocks(cols))
    params = cols * (4 if case.get("params") == "float32" else size)
    if case["op"] == "norm_forward":
        back = kept * 2 + 2 * values if case["kept"] else 0      # written, and read back as bf16 values
        return {"bytes": 2 * values * size + 2 * params + 8 * rows + back, "flops": 8 * values}
    if case["op"] == "norm_backward":
        x = kept if case["kept"] else values * size + 4 * rows
        return {"bytes": 2 * values * size + x + 4 * rows + params + 8 * cols, "flops": 14 * values}
    if case["op"] == "checkpoint":
        return {"bytes": 2 * values * size + 2 * kept, "flops": 5 * values}
    return {"bytes": 2 * values * size + kept + (4 * rows if case["goodness"] else 0), "flops": 12 * values}


# --- in 64 bits ---------------------------------------------------------------------------------------------------------
def _codes64(x, u):
    """The values that a checkpoint of x stands for, and its exponent bytes."""
    rows, cols = x.shape
    nb = _blocks(cols)
    most = torch.zeros(rows, nb, dtype=torch.float64, device="cuda")
    whole = cols // BLOCK
    if whole:
        most[:, :whole] = x[:, : whole * BLOCK].abs().reshape(rows, whole, BLOCK).amax(2)
    if whole < nb:
        most[:, whole] = x[:, whole * BLOCK:].abs().amax(1)
    none = most < 2.0**-100
    s = torch.ceil(torch.log2(torch.where(none, 127.0, most) / 127.0))
    s = torch.where(127.0 * torch.exp2(s) < most, s + 1, s)            # the logarithm's own rounding
    s = torch.where(127.0 * torch.exp2(s - 1) >= most, s - 1, s)
    s = torch.where(none, 0.0, s.clamp(max=121))
    step = torch.exp2(s).repeat_interleave(BLOCK, 1)[:, :cols]
    t = x / step
    if u is None:
        t = torch.round(t)
    else:
        t = torch.floor(t) + (u.double() < t - torch.floor(t)).double()
    t = torch.where(none.repeat_interleave(BLOCK, 1)[:, :cols], 0.0, t.clamp(-127, 127))
    return t * step, (s + 127).to(torch.uint8)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op in ("norm_backward", "act_backward", "weight_grad") and s["q"] is not None:
        cols = case["k"] if op == "weight_grad" else case["cols"]
        at = torch.arange(cols, device="cuda")
        kept = s["q"][:, at].double() * torch.pow(2.0, s["e"].double() - 127)[:, at // BLOCK]
    if op == "norm_forward":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        xh = (x - mean) * torch.rsqrt(var + EPS)
        out = {"y": s["weight"].double() * xh + s["bias"].double(), "mean": mean[:, 0], "rstd": torch.rsqrt(var + EPS)[:, 0]}
        if case["kept"]:
            out["kept"] = xh      # what the checkpoint stands for: its error is the rounding to 8 bits
        return out
    if op == "norm_backward":
        dy, r = s["dy"].double(), s["rstd"].double()[:, None]
        xh = kept if case["kept"] else r * (s["x"].double() - s["mean"].double()[:, None])
        h = dy * s["weight"].double()
        n = case["cols"]
        dx = r / n * (n * h - h.sum(1, keepdim=True) - xh * (h * xh).sum(1, keepdim=True))
        return {"dx": dx, "dweight": torch.linalg.vecdot(dy, xh, dim=0), "dbias": dy.sum(0)}
    if op == "checkpoint":
        u = _uniform(case["rows"], case["cols"], s["sr_seed"], s["tag"]) if case["stochastic"] else None
        v, e = _codes64(s["x"].double(), u)
        return {"back": v, "scale": e}
    if op == "act_backward":
        u, act = kept, case["act"]
        if act == "relu":
            a, d = torch.relu(u), (u > 0).double()
        elif act == "gelu":
            a, d = 0.5 * u * torch.erfc(-u / math.sqrt(2)), 0.5 * torch.erfc(-u / math.sqrt(2)) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
        elif act == "silu":
            a, d = u * torch.sigmoid(u), torch.sigmoid(u) + u * torch.sigmoid(u) * torch.sigmoid(-u)
        else:
            a, d = u, torch.ones_like(u)
        up = s["dy"].double()
        if case["goodness"]:
            up = up + 2 * a * s["coeff"].double()[:, None]
        return {"dx": up * d}
    dy = s["dy"].double()
    dw, db = torch.mm(dy.t(), kept), dy.sum(0)
    if case["affine"]:
        dw = dw * s["weight"].double() + torch.outer(db, s["bias"].double())
    return {"dweight": dw, "dbias": db}
