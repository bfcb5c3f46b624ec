"""Operators beside the block in 8-bit floating point, as cases that can be timed and compared.

    op "linear"         rows x [P, K] times weights [O, K] held as 8-bit integers with a scale for each row (channel of
                        the result): x is quantized to 8-bit integers with a scale for each row (token) on the way
    op "norm"           group norm with an activation of maps, channels last: N samples of S pixels of C channels in G
                        groups -> values in the type of x, and the statistics that the gradient needs
    op "norm_linear"    that norm, to the codes of a product with such weights: a normalised, activated map through a
                        pointwise layer, as it is served
    op "norm_backward"  the gradients of x, of the weight and of the bias of a norm
    op "clip"           the norm of all gradients of a model together, and the gradients scaled to at most a given norm,
                        into buffers that the optimizer reads

Codes of rows: s = max(amax / 127, 2^-126) with 1 / 127 rounded to f32, code = x * (1 / s) to the nearest whole number,
ties to even; every step is rounded to f32.
"""
import math
import random

import torch

own = False

EPS = 1e-5
CLIP_EPS = 1e-6
BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
ONE_127TH = 0.007874015718698502  # 1 / 127 as f32 has it
LEAST = 2.0 ** -126


def _case(name, **case):
    return dict(name=name, **case) if name else case


def _linear(name, P, K, O, dtype="bf16", bias=False):
    return _case(name, op="linear", P=P, K=K, O=O, dtype=dtype, bias=bias)


def _norm(name, N, S, C, G, op="norm", act="silu", dtype="bf16", weights="f32", O=0):
    return _case(name, op=op, N=N, S=S, C=C, G=G, act=act, dtype=dtype, weights=weights, O=O)


def _clip(name, tensors, values, dtype="bf16", out="same", max_norm=1.0, scale=1.0):
    return _case(name, op="clip", tensors=tensors, values=values, dtype=dtype, out=out, max_norm=max_norm, scale=scale)


def listed():
    return [
        # one token, or one pixel of a stream: the weights' bytes and every launch show
        _linear("linear_one_row", 1, 4096, 4096),
        # an ordinary batch or prompt
        _linear("linear_batch", 4096, 4096, 4096),
        # the largest: a prompt of several thousand rows through wide layers
        _linear("linear_large", 8192, 8192, 8192),
        # 64 maps of 7 x 7 pixels and one more, 960 channels (no multiple of 128), a bias, single precision
        _linear("linear_odd", 3137, 960, 1000, dtype="f32", bias=True),
        # one small map, as an image alone passes through a late stage
        _norm("norm_one_map", 1, 196, 256, 32),
        # a batch of the first maps of a residual network, half a group's values next to each other in memory
        _norm("norm_batch", 256, 3136, 64, 32, act="relu"),
        # one large image: few groups, each spread over a quarter of a million pixels
        _norm("norm_image", 1, 262144, 128, 32),
        # a served layer: a norm of 7 x 7 maps of 960 channels straight into a product, to the classes of a model
        _norm("norm_linear_odd", 65, 49, 960, 32, op="norm_linear", O=1000, dtype="f16", weights="f16"),
        # a training step on middle maps
        _norm("norm_backward_batch", 32, 3136, 256, 32, op="norm_backward"),
        # maps with sides that are multiples of nothing, groups of 23 channels, single precision
        _norm("norm_backward_odd", 7, 1739, 161, 7, op="norm_backward", act="none", dtype="f32"),
        # the gradients of a small network of blocks
        _clip("clip_small", 19, 1583616, dtype="f32"),
        # the gradients of a deep model, matrices in 16 bits and vectors in 32, scaled far down
        _clip("clip_large", 291, 400000003, dtype="mixed"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def _width(rng, high=8192):
    """Channels: mostly multiples of a vector, some odd."""
    if rng.random() < 0.7:
        return rng.choice([w for w in (64, 96, 128, 144, 256, 512, 576, 960, 1024, 2048, 2560, 4096, 5120, 8192) if w <= high])
    return _spread(rng, 33, (high - 1) // 2) * 2 - 1


def draw(rng):
    """One more case: 1 to 16384 rows of products, 1 to 256 maps of 1 to 262144 pixels of 8 to 2048 channels, 1 to 400
    gradients; every operator and type.  (Gradients of a ReLU jump at 0, where no two ways to round agree: the smooth
    activation and none stand for the gradients.)"""
    op = rng.choice(["linear", "linear", "linear", "norm", "norm", "norm_linear", "norm_backward", "norm_backward", "clip", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "linear":
        K, O = _width(rng), _width(rng)
        return _linear(None, _spread(rng, 1, min(16384, 8192 ** 3 / K / O)), K, O, dtype=dtype, bias=rng.random() < 0.4)
    if op == "clip":
        tensors = _spread(rng, 1, 400)
        return _clip(None, tensors, _spread(rng, 97 * tensors, 300000000), dtype=rng.choice(["mixed", dtype]), out=rng.choice(["same", "f32"]),
                     max_norm=rng.choice([0.1, 1.0, 1000.0]), scale=rng.choice([1.0, 0.125]))
    G = rng.choice([1, 4, 8, 16, 32, 32, rng.randint(2, 48)])
    C = G * _spread(rng, max(1, -(-8 // G)), 2048 // G)
    total = 256 * 3136 * 64 if op == "norm" else 32 * 3136 * 256
    N = _spread(rng, 1, 256)
    S = _spread(rng, max(1, 64 * G // C), max(1, 64 * G // C, min(262144, total // (N * C))))
    act = rng.choice(["none", "silu"] if op == "norm_backward" else ["none", "relu", "silu", "silu"])
    if op == "norm_linear":
        dtype = rng.choice(["bf16", "f16"])
    return _norm(None, N, S, C, G, op=op, act=act, dtype=dtype, weights=rng.choice(["f32", dtype]),
                 O=_width(rng, 2048) if op == "norm_linear" else 0)


# ---- the plain forms ----

def _codes(x):
    """rows (f32) -> whole numbers of -127 to 127 (as f32), the rows' scales [rows, 1]"""
    s = (x.abs().amax(1, keepdim=True) * ONE_127TH).clamp_min(LEAST)
    return torch.round(x * (1.0 / s)), s


def _times_weights(s, x):
    c = s["case"]
    q, scale = _codes(x)
    y = (q @ s["w"][:, :x.shape[1]].to(torch.float32).t()) * (scale * s["w_scales"])
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[c["dtype"]])


def _act(z, act):
    return z if act == "none" else z.clamp_min(0.0) if act == "relu" else z / (1.0 + torch.exp(-z))


def _groups(t, c):
    return t.view(c["N"], c["S"], c["G"], c["C"] // c["G"])


def _affine(s):
    c = s["case"]
    return (s[k].to(torch.float32).view(1, 1, c["G"], -1) for k in ("weight", "shift"))


def _normalise(s):
    """-> the activated values [N S, C] in f32, means and reciprocal deviations [2, N, G]"""
    c = s["case"]
    w, b = _affine(s)
    x = _groups(s["x"].to(torch.float32), c)
    mean = x.mean((1, 3), keepdim=True)
    x = x - mean
    rstd = torch.rsqrt(x.square().mean((1, 3), keepdim=True) + EPS)
    y = _act(x * rstd * w + b, c["act"])
    return y.view(-1, c["C"]), torch.stack([mean.view(c["N"], c["G"]), rstd.view(c["N"], c["G"])])


def _run_norm(s):
    y, stats = _normalise(s)
    return [y.to(s["x"].dtype), stats]


def _run_norm_linear(s):
    return _times_weights(s, _normalise(s)[0])


def _run_norm_backward(s):
    c = s["case"]
    w, b = _affine(s)
    mean, rstd = (t[:, None, :, None] for t in s["stats"])
    x = (_groups(s["x"].to(torch.float32), c) - mean) * rstd
    dz = _groups(s["dy"].to(torch.float32), c)
    if c["act"] == "silu":
        z = x * w + b
        p = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * (p * (1.0 + z * (1.0 - p)))
    a = dz * w
    dx = rstd * (a - a.mean((1, 3), keepdim=True) - x * (a * x).mean((1, 3), keepdim=True))
    return [dx.view(-1, c["C"]).to(s["x"].dtype), (dz * x).sum((0, 1)).view(-1), dz.sum((0, 1)).view(-1)]


def _run_clip(s):
    c = s["case"]
    total = torch.stack([g.to(torch.float32).square().sum(dtype=torch.float64) for g in s["grads"]]).sum()
    norm = c["scale"] * total.sqrt()
    factor = (c["scale"] * (c["max_norm"] / (norm + CLIP_EPS)).clamp_max(1.0)).to(torch.float32)
    [o.copy_(g.to(torch.float32) * factor) for g, o in zip(s["grads"], s["outs"])]
    return [norm.to(torch.float32).view(1), *s["out_flats"]]


_PLAIN = {"linear": lambda s: _times_weights(s, s["x"].to(torch.float32)), "norm": _run_norm, "norm_linear": _run_norm_linear,
          "norm_backward": _run_norm_backward, "clip": _run_clip}


# ---- the framework's calls ----

def _run_own(s):
    from paper_1905_10830_amd import binding as fmtc

    c = s["case"]
    if c["op"] == "linear":
        return fmtc.i8_linear(s["x"], s["w_handle"], bias=s["bias"])
    if c["op"] == "clip":
        return [s["list_handle"].clip(c["max_norm"], scale=c["scale"], eps=CLIP_EPS), *s["out_flats"]]
    act = {"none": fmtc.ACT_NONE, "relu": fmtc.ACT_RELU, "silu": fmtc.ACT_SILU}[c["act"]]
    if c["op"] == "norm":
        y, stats = fmtc.group_norm(s["x"], c["G"], s["weight"], s["shift"], rows_per_sample=c["S"], act=act, eps=EPS, stats=True)
        return [y, stats]
    if c["op"] == "norm_linear":
        n, _ = fmtc.group_norm(s["x"], c["G"], s["weight"], s["shift"], rows_per_sample=c["S"], act=act, eps=EPS,
                               out=fmtc.i8_empty(c["N"] * c["S"], c["C"]))
        return fmtc.i8_matmul(n, s["w_handle"], bias=s["bias"], dtype=DTYPES[c["dtype"]])
    return list(fmtc.group_norm_backward(s["dy"], s["x"], s["stats"], c["G"], s["weight"], s["shift"], rows_per_sample=c["S"], act=act))


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---- inputs ----

def _activations(g, P, C):
    """Rows of a network's activations: channels of different size, a few of them large, rows of different size."""
    x = torch.randn((P, C), generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
    x *= torch.where(torch.rand(C, generator=g, device="cuda") < 0.005, 12.0, 1.0)
    return x.mul_(torch.exp(0.3 * torch.randn((P, 1), generator=g, device="cuda")))


def _add_weights(s, g, O, K, bias):
    """Weights as a program keeps them: codes with zeros behind the depth, a scale for each row."""
    w = torch.randn((O, K), generator=g, device="cuda") * (0.02 * torch.exp(0.3 * torch.randn((O, 1), generator=g, device="cuda")))
    q, scale = _codes(w)
    s["w"] = torch.nn.functional.pad(q, (0, -K % BLOCK)).to(torch.int8)
    s["w_scales"] = scale.view(-1)
    s["bias"] = 0.1 * torch.randn(O, generator=g, device="cuda") if bias else None
    if own:
        from paper_1905_10830_amd import binding as fmtc

        s["w_handle"] = fmtc.I8(s["w"], s["w_scales"], K)
    return s


def _sizes(c):
    """Values of each gradient: matrices of different size, and a vector after every second one."""
    rng = random.Random(c["tensors"] * 1000003 + c["values"])
    part = [math.exp(rng.gauss(0.0, 1.0)) * (0.001 if i % 3 == 2 else 1.0) for i in range(c["tensors"])]
    n = [max(1, int(c["values"] * p / sum(part))) for p in part]
    n[0] += max(0, c["values"] - sum(n))
    return n


def _flat_views(c, dtype, n):
    """One buffer for each type, and the gradients as views of it: matrices in 16 bits and vectors in 32 where types are mixed."""
    kinds = [("f32" if i % 3 == 2 else "bf16") if dtype == "mixed" else dtype for i in range(len(n))]
    flats = {k: torch.zeros(sum(v for v, t in zip(n, kinds) if t == k), dtype=DTYPES[k], device="cuda") for k in sorted(set(kinds))}
    views, at = [], dict.fromkeys(flats, 0)
    for v, k in zip(n, kinds):
        views.append(flats[k][at[k]:at[k] + v])
        at[k] += v
    return list(flats.values()), views


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "linear":
        s["x"] = _activations(g, c["P"], c["K"]).to(DTYPES[c["dtype"]])
        return _add_weights(s, g, c["O"], c["K"], c["bias"])
    if c["op"] == "clip":
        n = _sizes(c)
        flats, s["grads"] = _flat_views(c, c["dtype"], n)
        for f in flats:
            f.copy_(torch.randn(f.numel(), generator=g, device="cuda", dtype=torch.float32 if f.dtype == torch.float32 else torch.bfloat16))
            f.mul_(1e-3)
        s["out_flats"], s["outs"] = _flat_views(c, "f32" if c["out"] == "f32" else c["dtype"], n)
        if own:
            from paper_1905_10830_amd import binding as fmtc

            s["list_handle"] = fmtc.Tensors(s["grads"], out=s["outs"])
        return s
    t, wt = DTYPES[c["dtype"]], DTYPES[c["weights"]]
    x = _activations(g, c["N"] * c["S"], c["C"])
    s["x"] = x.add_(torch.randn(c["C"], generator=g, device="cuda")).to(t)
    s["weight"] = (1.0 + 0.2 * torch.randn(c["C"], generator=g, device="cuda")).to(wt)
    s["shift"] = (0.2 * torch.randn(c["C"], generator=g, device="cuda")).to(wt)
    if c["op"] == "norm_linear":
        return _add_weights(s, g, c["O"], c["C"], True)
    if c["op"] == "norm_backward":  # stats as the forward pass left them
        s["dy"] = (1e-3 * torch.randn((c["N"] * c["S"], c["C"]), generator=g, device="cuda")).to(t)
        s["stats"] = _normalise(s)[1]
    return s


def work(case):
    c = case
    if c["op"] == "linear":
        P, K, O, size = c["P"], c["K"], c["O"], SIZE[c["dtype"]]
        return {"bytes": size * P * K + O * K + 4 * O + size * P * O + (4 * O if c["bias"] else 0), "flops": 2 * P * K * O}
    if c["op"] == "clip":
        n = _sizes(c)
        kinds = [("f32" if i % 3 == 2 else "bf16") if c["dtype"] == "mixed" else c["dtype"] for i in range(len(n))]
        return {"bytes": sum(v * (SIZE[k] + (4 if c["out"] == "f32" else SIZE[k])) for v, k in zip(n, kinds)) + 4, "flops": 3 * sum(n)}
    n, size, params = c["N"] * c["S"] * c["C"], SIZE[c["dtype"]], 2 * SIZE[c["weights"]] * c["C"]
    stats = 8 * c["N"] * c["G"]
    if c["op"] == "norm":
        return {"bytes": 2 * size * n + params + stats, "flops": 10 * n}
    if c["op"] == "norm_backward":
        return {"bytes": 3 * size * n + params + stats + 8 * c["C"], "flops": 25 * n}
    P, O = c["N"] * c["S"], c["O"]
    return {"bytes": size * n + params + O * c["C"] + 8 * O + size * P * O, "flops": 2 * P * c["C"] * O + 10 * n}


# ---- the definitions, in 64 bits ----

def _exact_f32(v):
    """A number in 64 bits to the nearest of 32 bits: the definition of the codes has such steps."""
    return v.to(torch.float32).to(torch.float64)


def _exact_product(s, x, depth):
    largest = torch.max(torch.abs(x), 1).values
    scale = torch.maximum(_exact_f32(largest * ONE_127TH), torch.full_like(largest, LEAST))
    codes = torch.round(_exact_f32(x * _exact_f32(torch.reciprocal(scale))[:, None]))
    y = torch.matmul(codes, s["w"][:, :depth].double().t()) * scale[:, None] * s["w_scales"].double()
    return y if s["bias"] is None else y + s["bias"].double()


def _exact_norm(s):
    c = s["case"]
    D, count = c["C"] // c["G"], c["S"] * (c["C"] // c["G"])
    owner = torch.arange(c["C"], device="cuda") // D
    x = s["x"].double().reshape(c["N"], c["S"], c["C"])
    mean = torch.sum(torch.sum(x, 1).reshape(c["N"], c["G"], D), 2) / count
    x = x - mean[:, owner][:, None]
    var = torch.sum(torch.sum(x * x, 1).reshape(c["N"], c["G"], D), 2) / count
    rstd = 1.0 / torch.sqrt(var + EPS)
    z = x.mul_((rstd[:, owner] * s["weight"].double())[:, None]).add_(s["shift"].double())
    if c["act"] == "relu":
        z = torch.maximum(z, torch.zeros_like(z))
    elif c["act"] == "silu":
        z = z * torch.sigmoid(z)
    return z.reshape(-1, c["C"]), torch.stack([mean, rstd])


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "linear":
        return _exact_product(s, s["x"].double(), c["K"])
    if c["op"] == "norm":
        return list(_exact_norm(s))
    if c["op"] == "norm_linear":
        return _exact_product(s, _exact_norm(s)[0], c["C"])
    if c["op"] == "clip":
        norm = c["scale"] * math.sqrt(sum(float(torch.dot(p, p)) for g in s["grads"] for p in (g.double(),)))
        factor = c["scale"] * min(1.0, c["max_norm"] / (norm + CLIP_EPS))
        flats = [torch.zeros(f.numel(), dtype=torch.float64, device="cuda") for f in s["out_flats"]]
        kinds, at = [f.dtype for f in s["out_flats"]], [0] * len(flats)
        for g, o in zip(s["grads"], s["outs"]):
            k = kinds.index(o.dtype)
            flats[k][at[k]:at[k] + g.numel()] = factor * g.double()
            at[k] += g.numel()
        return [torch.full((1,), norm, dtype=torch.float64, device="cuda"), *flats]
    D = c["C"] // c["G"]
    owner = torch.arange(c["C"], device="cuda") // D
    mean, rstd = s["stats"].double()
    w = s["weight"].double()
    r = rstd[:, owner][:, None]
    x = (s["x"].double().reshape(c["N"], c["S"], c["C"]) - mean[:, owner][:, None]) * r
    dz = s["dy"].double().reshape(c["N"], c["S"], c["C"])
    if c["act"] == "silu":
        z = x * w + s["shift"].double()
        p = torch.sigmoid(z)
        dz = dz * (p + z * p * torch.sigmoid(-z))
    d_b, d_w = torch.sum(dz, 1), torch.sum(dz * x, 1)
    # dx = rstd (w dz - (sum of w dz + x^ sum of w dz x^) / count), the sums over a sample's group
    sums = [torch.sum((t * w).reshape(c["N"], c["G"], D), 2)[:, owner][:, None] / (c["S"] * D) for t in (d_b, d_w)]
    dx = r * (dz * w - sums[0] - x * sums[1])
    return [dx.reshape(-1, c["C"]), torch.sum(d_w, 0), torch.sum(d_b, 0)]
