"""The operators of a block of a network in 8-bit floating point, as cases that can be timed and compared.

A block reads a stream h of P rows (pixels or tokens) of C channels, multiplies normalised rows by weights and adds its
gated output back to the stream.  The rows, the weights and the gradients that enter a matrix product are held as 8-bit
floating point numbers ("codes") with a scale for each block of 128; everything else is bf16, f16 or f32.  The cases
stand for the calls that a program makes for it:

    op "quantize"       values [P, C] -> codes and scales, by rows (1 x 128 blocks), by rows and by columns (128 x 1
                        blocks, transposed, for a product over the rows), or as weights (128 x 128 blocks)
    op "product"        codes [P, K] times codes of weights [O, K] -> y [P, O], with a bias or without one
    op "backward"       the gradient of a product: dy [P, O] -> dx [P, K], dw [O, K], dbias [O]; dy is quantized on the
                        way, the weights and x are held as codes, laid out for these products
    op "norm"           between two blocks: u = norm(y) w_post, h' = skip h + scale gate u, n = norm(h') w_pre, n in
                        the type of h or as codes with scales
    op "norm_backward"  the gradients of y, h, w_post, w_pre and the gate

Layouts: codes are [rows, depth rounded up to 128] with zeros behind the depth, scales [blocks along the depth, blocks
of rows]; scales are f32, or powers of two as 8-bit exponents ("e8m0").  A gate has one row for `rows_per_gate` rows of
the stream.
"""
import math

import torch

own = False

EPS = 1e-6
BLOCK = 128
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}          # both are 1.75 times a power of two
EXPONENT = {"e4m3": 8, "e5m2": 15}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def _case(name, **case):
    return dict(name=name, **case) if name else case


def _quantize(name, P, C, dtype="bf16", fmt="e4m3", scales="f32", blocks="rows"):
    return _case(name, op="quantize", P=P, C=C, dtype=dtype, fmt=fmt, scales=scales, blocks=blocks)


def _product(name, P, K, O, dtype="bf16", scales="f32", bias=False):
    return _case(name, op="product", P=P, K=K, O=O, dtype=dtype, scales=scales, bias=bias)


def _backward(name, P, K, O, dtype="bf16", fmt="e4m3", scales="f32", bias=False):
    return _case(name, op="backward", P=P, K=K, O=O, dtype=dtype, fmt=fmt, scales=scales, bias=bias)


def _norm(name, P, C, op="norm", dtype="bf16", weights="f32", rows_per_gate=0, skip=1.0, scale=1.0, codes=False, scales="f32"):
    return _case(name, op=op, P=P, C=C, dtype=dtype, weights=weights, rows_per_gate=rows_per_gate, skip=skip, scale=scale,
                 codes=codes, scales=scales)


def listed():
    return [
        # one token, or one pixel of a stream: the time to read the weights and every launch show
        _product("product_one_row", 1, 4096, 4096),
        # a few requests served together, wide layers, power-of-two scales
        _product("product_few_rows", 13, 8192, 8192, scales="e8m0"),
        # an ordinary batch of a training step or a prompt
        _product("product_batch", 4096, 4096, 4096),
        # the largest: a prompt of several thousand rows through wide layers
        _product("product_large", 8192, 8192, 8192, scales="e8m0"),
        # 64 maps of 7 x 7 pixels and one more, 960 channels (no multiple of 128), a bias, another type
        _product("product_odd", 3137, 960, 1000, dtype="f16", bias=True),
        # the gradient of that ordinary batch
        _backward("backward_batch", 4096, 4096, 4096),
        # sizes that are multiples of nothing, gradients with more range and less precision
        _backward("backward_odd", 3001, 960, 577, fmt="e5m2", scales="e8m0", bias=True),
        # activations of a training step, for the product and for the weights' gradient
        _quantize("quantize_both", 8192, 4096, blocks="both"),
        # a handful of rows of an odd width, single precision, power-of-two scales
        _quantize("quantize_small", 77, 1000, dtype="f32", scales="e8m0"),
        # between two blocks, one token: straight to the codes of the next product
        _norm("norm_one_row", 1, 4096, rows_per_gate=1, codes=True),
        # between two blocks, a training step or a long prompt, one gate for all rows
        _norm("norm_large", 16384, 4096, rows_per_gate=16384, scale=0.5),
        # its gradient, eight samples with a gate each
        _norm("norm_backward_large", 8192, 4096, op="norm_backward", rows_per_gate=1024, skip=0.9),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, high=8192):
    """Channels: mostly multiples of a vector, some odd."""
    if rng.random() < 0.7:
        return rng.choice([w for w in (64, 96, 128, 144, 256, 512, 576, 960, 1024, 2048, 2560, 4096, 5120, 8192) if w <= high])
    return _spread(rng, 33, (high - 1) // 2) * 2 - 1


def draw(rng):
    """One more case: 1 to 16384 rows, 64 to 8192 channels, every operator, type and kind of scale."""
    op = rng.choice(["quantize", "product", "product", "product", "backward", "norm", "norm", "norm_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    scales = rng.choice(["f32", "e8m0"])
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    if op == "product":
        K, O = _width(rng), _width(rng)
        return _product(None, _spread(rng, 1, min(16384, 8192 ** 3 / K / O)), K, O, dtype=dtype, scales=scales, bias=rng.random() < 0.4)
    if op == "backward":
        K, O = _width(rng, 5120), _width(rng, 5120)
        return _backward(None, _spread(rng, 16, min(16384, 4096 ** 3 / K / O)), K, O, dtype=dtype, fmt=fmt, scales=scales, bias=rng.random() < 0.4)
    C = _width(rng)
    if op == "quantize":
        return _quantize(None, _spread(rng, 1, min(16384, 8192 * 4096 // C)), C, dtype=dtype, fmt=fmt, scales=scales,
                         blocks=rng.choice(["rows", "both", "weights"]))
    P = _spread(rng, 1, min(16384, 8192 * 4096 // C))
    return _norm(None, P, C, op=op, dtype=dtype, weights=rng.choice(["f32", dtype]),
                 rows_per_gate=rng.choice([0, 1, P, max(1, P // 8), rng.randint(1, P)]),
                 skip=rng.choice([1.0, 0.9]), scale=rng.choice([1.0, 0.5]), codes=op == "norm" and rng.random() < 0.5, scales=scales)


# ---- the plain forms ----

def _up(n):
    return -(-n // BLOCK) * BLOCK


def _scale_of(amax, fmt, kind):
    """-> (scale as f32, scale as it is held).  f32: amax over the largest code; e8m0: the next power of two."""
    if kind == "f32":
        s = (amax / LARGEST[fmt]).clamp_min(2.0 ** -126)
        return s, s
    e = (((amax.view(torch.int32) + 0x1fffff) >> 23) - EXPONENT[fmt]).clamp(1, 254)
    return (e << 23).view(torch.float32), e.to(torch.uint8).view(torch.float8_e8m0fnu)


def _amax(x, dims):
    a = x.abs()
    return torch.where(torch.isfinite(a), a, torch.zeros_like(a)).amax(dims)


def _encode(x, fmt, kind, block_rows=1):
    """values [R, D] (f32) -> codes [R, D up to 128], scales [D / 128, R / block_rows]."""
    R, D = x.shape
    Rp, Dp = -(-R // block_rows) * block_rows, _up(D)
    if (Rp, Dp) != (R, D):
        x = torch.nn.functional.pad(x, (0, Dp - D, 0, Rp - R))
    x = x.view(Rp // block_rows, block_rows, Dp // BLOCK, BLOCK)
    s, held = _scale_of(_amax(x, (1, 3)), fmt, kind)
    codes = (x * (1.0 / s)[:, None, :, None]).to(CODES[fmt]).view(Rp, Dp)
    return codes[:R], held.t().contiguous()


def _decode(codes, scales, depth):
    """-> the values [R, depth] (f32) that codes stand for."""
    R, Dp = codes.shape
    s = scales.to(torch.float32).t()
    x = codes.to(torch.float32).view(R, Dp // BLOCK, BLOCK)
    s = s if len(s) == R else s.repeat_interleave(BLOCK, 0)[:R]
    return (x * s[:, :, None]).view(R, Dp)[:, :depth]


def _run_quantize(s):
    c, x = s["case"], s["x"].to(torch.float32)
    if c["blocks"] == "weights":
        return [*_encode(x, c["fmt"], c["scales"], BLOCK), *_encode(x.t().contiguous(), c["fmt"], c["scales"], BLOCK)]
    out = [*_encode(x, c["fmt"], c["scales"])]
    if c["blocks"] == "both":
        out += _encode(x.t().contiguous(), c["fmt"], c["scales"])
    return out


def _run_product(s):
    c = s["case"]
    y = _decode(*s["x"], c["K"]) @ _decode(*s["w"], c["K"]).t()
    if c["bias"]:
        y = y + s["bias"]
    return y.to(DTYPES[c["dtype"]])


def _run_backward(s):
    c = s["case"]
    dy = s["dy"].to(torch.float32)
    dx = _decode(*_encode(dy, c["fmt"], c["scales"]), c["O"]) @ _decode(*s["w_t"], c["O"]).t()
    dw = _decode(*_encode(dy.t().contiguous(), c["fmt"], c["scales"]), c["P"]) @ _decode(*s["x_t"], c["P"]).t()
    return [dx.to(DTYPES[c["dtype"]]), dw] + ([dy.sum(0)] if c["bias"] else [])


def _gate_rows(s):
    """-> scale * gate as it meets each row of the stream, f32."""
    c = s["case"]
    if s["gate"] is None:
        return torch.tensor(c["scale"], dtype=torch.float32, device="cuda")
    g = s["gate"].to(torch.float32) * c["scale"]
    return g if len(g) == 1 else g.repeat_interleave(c["rows_per_gate"], 0)[:c["P"]]


def _run_norm(s):
    c = s["case"]
    y, h = s["y"].to(torch.float32), s["h"].to(torch.float32)
    r_y = torch.rsqrt(y.square().mean(1, keepdim=True) + EPS)
    h = c["skip"] * h + _gate_rows(s) * (y * r_y * s["w_post"].to(torch.float32))
    r_h = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    n = h * r_h * s["w_pre"].to(torch.float32)
    stats = torch.stack([r_y[:, 0], r_h[:, 0]])
    n = _encode(n, "e4m3", c["scales"]) if c["codes"] else [n.to(s["h"].dtype)]
    return [h.to(s["h"].dtype), *n, stats]


def _run_norm_backward(s):
    c, t = s["case"], s["h"].dtype
    y, h, dn = (s[k].to(torch.float32) for k in ("y", "h", "dn"))
    r_y, r_h = s["stats"][0][:, None], s["stats"][1][:, None]
    w_post, w_pre, gate = s["w_post"].to(torch.float32), s["w_pre"].to(torch.float32), _gate_rows(s)
    y, h = y * r_y, h * r_h
    a = dn * w_pre
    dh = s["dh"].to(torch.float32) + r_h * (a - h * (a * h).mean(1, keepdim=True))
    du = gate * dh
    b = du * w_post
    dy = r_y * (b - y * (b * y).mean(1, keepdim=True))
    out = [dy.to(t), (c["skip"] * dh).to(t), (du * y).sum(0), (dn * h).sum(0)]
    if s["gate"] is not None:
        each = c["scale"] * dh * y * w_post
        G, R = len(s["gate"]), c["rows_per_gate"]
        if G * R != len(each):
            each = torch.nn.functional.pad(each, (0, 0, 0, G * R - len(each)))
        out.append(each.view(G, R, -1).sum(1))
    return out


_PLAIN = {"quantize": _run_quantize, "product": _run_product, "backward": _run_backward, "norm": _run_norm,
          "norm_backward": _run_norm_backward}


# ---- the framework's calls ----

def _own_f8(fmtc, pair, depth, block_rows=1):
    return fmtc.F8(pair[0], pair[1], depth, block_rows)


def _own_kinds(fmtc, c):
    return dict(fmt=fmtc.E5M2 if c.get("fmt") == "e5m2" else fmtc.E4M3,
                scales=fmtc.SCALE_E8M0 if c["scales"] == "e8m0" else fmtc.SCALE_F32)


def _run_own(s):
    from paper_1905_10830_amd import binding as fmtc

    c = s["case"]
    if c["op"] == "quantize":
        got = fmtc.f8_quantize(s["x"], by_rows=True, by_cols=c["blocks"] != "rows",
                               block_rows=BLOCK if c["blocks"] == "weights" else 1, **_own_kinds(fmtc, c))
        return [t for q in got if q is not None for t in (q.codes, q.scales)]
    if c["op"] == "product":
        return fmtc.f8_matmul(_own_f8(fmtc, s["x"], c["K"]), _own_f8(fmtc, s["w"], c["K"], BLOCK), bias=s["bias"], dtype=DTYPES[c["dtype"]])
    if c["op"] == "backward":
        dx, dw, dbias = fmtc.f8_matmul_backward(s["dy"], _own_f8(fmtc, s["w_t"], c["O"], BLOCK), _own_f8(fmtc, s["x_t"], c["P"]),
                                                bias=c["bias"], **_own_kinds(fmtc, c))
        return [dx, dw] + ([dbias] if c["bias"] else [])
    gate = dict(gate=s["gate"], rows_per_gate=c["rows_per_gate"], skip=c["skip"], scale=c["scale"])
    if c["op"] == "norm":
        n = fmtc.f8_empty(c["P"], c["C"], scales=_own_kinds(fmtc, c)["scales"], device="cuda") if c["codes"] else None
        h, n, stats = fmtc.block_norm(s["y"], s["h"], s["w_post"], s["w_pre"], eps=EPS, n_out=n, stats=True, **gate)
        return [h, *((n.codes, n.scales) if c["codes"] else (n,)), stats]
    dy, dh, dw_post, dw_pre, dgate = fmtc.block_norm_backward(s["dn"], s["dh"], s["y"], s["h"], s["stats"], s["w_post"], s["w_pre"], **gate)
    return [dy, dh, dw_post, dw_pre] + ([dgate] if dgate is not None else [])


def run(state):
    return _run_own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---- inputs ----

def _activations(g, P, C):
    """Rows of a network's activations: channels of different size, a few of them large, rows of different size."""
    x = torch.randn((P, C), generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
    x *= torch.where(torch.rand(C, generator=g, device="cuda") < 0.005, 12.0, 1.0)
    return x.mul_(torch.exp(0.3 * torch.randn((P, 1), generator=g, device="cuda")))


def _weights(g, O, K):
    return torch.randn((O, K), generator=g, device="cuda") * (0.02 * torch.exp(0.3 * torch.randn((O, 1), generator=g, device="cuda")))


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "quantize":
        x = _weights(g, c["P"], c["C"]) if c["blocks"] == "weights" else _activations(g, c["P"], c["C"])
        return s | {"x": x.to(DTYPES[c["dtype"]])}
    if c["op"] == "product":
        s["x"] = _encode(_activations(g, c["P"], c["K"]), "e4m3", c["scales"])
        s["w"] = _encode(_weights(g, c["O"], c["K"]), "e4m3", c["scales"], BLOCK)
        s["bias"] = 0.1 * torch.randn(c["O"], generator=g, device="cuda") if c["bias"] else None
        return s
    if c["op"] == "backward":
        s["dy"] = (1e-3 * _activations(g, c["P"], c["O"])).to(DTYPES[c["dtype"]])
        s["w_t"] = _encode(_weights(g, c["O"], c["K"]).t().contiguous(), "e4m3", c["scales"], BLOCK)
        s["x_t"] = _encode(_activations(g, c["P"], c["K"]).t().contiguous(), "e4m3", c["scales"])
        return s
    P, C, t, wt = c["P"], c["C"], DTYPES[c["dtype"]], DTYPES[c["weights"]]
    s["y"] = _activations(g, P, C).to(t)
    s["h"] = (2.0 * _activations(g, P, C)).to(t)
    s["w_post"] = (1.0 + 0.2 * torch.randn(C, generator=g, device="cuda")).to(wt)
    s["w_pre"] = (1.0 + 0.2 * torch.randn(C, generator=g, device="cuda")).to(wt)
    R = c["rows_per_gate"]
    s["gate"] = torch.randn((-(-P // R), C), generator=g, device="cuda").to(wt) if R else None
    if c["op"] == "norm_backward":  # h is the stream behind the block here, stats what the forward pass left
        s["dn"] = (1e-3 * torch.randn((P, C), generator=g, device="cuda")).to(t)
        s["dh"] = (1e-3 * torch.randn((P, C), generator=g, device="cuda")).to(t)
        s["stats"] = torch.stack([torch.rsqrt(s[k].to(torch.float32).square().mean(1) + EPS) for k in ("y", "h")])
    return s


def work(case):
    c = case
    if c["op"] in ("product", "backward"):
        P, K, O, size, scale = c["P"], c["K"], c["O"], SIZE[c["dtype"]], 4 if c["scales"] == "f32" else 1
        bias = 4 * O if c["bias"] else 0
        if c["op"] == "product":
            blocks = -(-K // BLOCK)
            return {"bytes": P * K + O * K + scale * blocks * (P + -(-O // BLOCK)) + size * P * O + bias, "flops": 2 * P * K * O}
        rows = scale * (-(-O // BLOCK) * -(-K // BLOCK) + -(-P // BLOCK) * K)
        return {"bytes": size * P * O + O * K + P * K + rows + size * P * K + 4 * O * K + bias, "flops": 4 * P * K * O}
    P, C, size = c["P"], c["C"], SIZE[c["dtype"]]
    codes = P * C + (4 if c["scales"] == "f32" else 1) * P * -(-C // BLOCK)
    if c["op"] == "quantize":
        times = 1 if c["blocks"] == "rows" else 2
        return {"bytes": size * P * C + times * codes, "flops": 4 * times * P * C}
    gates = -(-P // c["rows_per_gate"]) * C if c["rows_per_gate"] else 0
    params = SIZE[c["weights"]] * (2 * C + gates)
    if c["op"] == "norm":
        return {"bytes": 3 * size * P * C + (codes if c["codes"] else size * P * C) + 8 * P + params, "flops": 12 * P * C}
    return {"bytes": 6 * size * P * C + 8 * P + params + 4 * (2 * C + gates), "flops": 30 * P * C}


# ---- the definitions, in 64 bits ----

def _exact_power(e):
    """2 to whole powers, as numbers in 64 bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_round(v, fmt):
    """The nearest number of the 8-bit format, ties to the even one; |v| is at most the largest."""
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = torch.frexp(v.abs())
    step = _exact_power((e - 1).clamp_min(least) - bits)
    return torch.round(v / step) * step


def _exact_codes(x, fmt, kind, block_rows=1):
    R, D = x.shape
    blocks = torch.zeros((-(-R // block_rows) * block_rows, _up(D)), dtype=torch.float64, device=x.device)
    blocks[:R, :D] = x
    blocks = blocks.view(blocks.shape[0] // block_rows, block_rows, -1, BLOCK)
    amax = blocks.abs().amax((1, 3))
    s = (amax / LARGEST[fmt]).clamp_min(2.0 ** -126)
    if kind == "f32":
        s = s.to(torch.float32).to(torch.float64)
    else:
        m, e = torch.frexp(s)
        s = _exact_power(torch.where(m > 0.5, e, e - 1))
    v = (blocks / s[:, None, :, None]).clamp(-LARGEST[fmt], LARGEST[fmt])
    return _exact_round(v, fmt).view(-1, _up(D))[:R], s


def _exact_values(pair, depth):
    codes, scales = pair[0].to(torch.float64), pair[1].to(torch.float64)
    rows = torch.arange(codes.shape[0], device="cuda")
    if scales.shape[1] != codes.shape[0]:
        rows = rows // BLOCK
    cols = torch.arange(codes.shape[1], device="cuda") // BLOCK
    return (codes * scales[cols][:, rows].t())[:, :depth]


def _exact_again(x, fmt, kind):
    """Rows of x as their codes stand for them."""
    q, s = _exact_codes(x, fmt, kind)
    return (q.view(len(x), -1, BLOCK) * s[:, :, None]).view(len(x), -1)[:, :x.shape[1]]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f8 = lambda x, fmt, block_rows=1: [(q, k.t()) for q, k in [_exact_codes(x, fmt, c["scales"], block_rows)]][0]  # noqa: E731
    if c["op"] == "quantize":
        x, block_rows = s["x"].double(), BLOCK if c["blocks"] == "weights" else 1
        return [*f8(x, c["fmt"], block_rows), *(f8(x.t(), c["fmt"], block_rows) if c["blocks"] != "rows" else ())]
    if c["op"] == "product":
        y = torch.matmul(_exact_values(s["x"], c["K"]), _exact_values(s["w"], c["K"]).t())
        return y if s["bias"] is None else y + s["bias"].double()
    if c["op"] == "backward":
        dy = s["dy"].double()
        dx = torch.matmul(_exact_again(dy, c["fmt"], c["scales"]), _exact_values(s["w_t"], c["O"]).t())
        dw = torch.matmul(_exact_again(dy.t(), c["fmt"], c["scales"]), _exact_values(s["x_t"], c["P"]).t())
        return [dx, dw] + ([dy.sum(0)] if c["bias"] else [])
    y, h, w_post, w_pre = (s[k].double() for k in ("y", "h", "w_post", "w_pre"))
    owner = torch.arange(c["P"], device="cuda") // max(1, c["rows_per_gate"])
    gate = c["scale"] * (s["gate"].double()[owner] if s["gate"] is not None else torch.ones_like(y))
    if c["op"] == "norm":
        i_y = 1.0 / torch.sqrt(torch.sum(y * y, 1) / c["C"] + EPS)
        h = c["skip"] * h + gate * w_post * y * i_y[:, None]
        i_h = 1.0 / torch.sqrt(torch.sum(h * h, 1) / c["C"] + EPS)
        n = w_pre * h * i_h[:, None]
        return [h, *(f8(n, "e4m3") if c["codes"] else (n,)), torch.stack([i_y, i_h])]
    i_y, i_h = s["stats"].double()[:, :, None]
    dn, dt = s["dn"].double(), s["dh"].double()
    y, h = y * i_y, h * i_h
    # d(v / rms(v)) = (dv - v^ <dv, v^> / C) / rms(v), once for the stream and once for the block's output
    dt = dt + i_h * (dn * w_pre - h * (torch.sum(dn * w_pre * h, 1, True) / c["C"]))
    dv = gate * dt * w_post
    out = [i_y * (dv - y * (torch.sum(dv * y, 1, True) / c["C"])), c["skip"] * dt,
           torch.sum(gate * dt * y, 0), torch.sum(dn * h, 0)]
    if s["gate"] is not None:
        out.append(torch.zeros(s["gate"].shape, dtype=torch.float64, device="cuda").index_add_(0, owner, c["scale"] * dt * y * w_post))
    return out
