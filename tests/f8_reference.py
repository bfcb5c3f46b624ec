"""Plain implementations, in 64 bits on the CPU, of the block operators: what their tests hold the kernels against."""
import torch

BLOCK = 128
LARGEST = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}


def blocks(n):
    return -(-n // BLOCK)


def _f32(x):
    return x.to(torch.float32).to(torch.float64)


def round_codes(v, dtype):
    """The nearest number of the 8-bit format (64 bits in and out), ties to even; infinities: NaN in E4M3."""
    bits, least = (3, -6) if dtype == torch.float8_e4m3fn else (2, -14)
    finite = torch.isfinite(v)
    a = torch.where(finite, v, torch.zeros_like(v))
    _, e = torch.frexp(a.abs())
    step = torch.ldexp(torch.ones_like(a), (e - 1).clamp_min(least) - bits)
    r = torch.round(a / step) * step
    bad = v if dtype == torch.float8_e5m2 else torch.full_like(v, float("nan"))
    return torch.where(finite, r, bad)


def quantize(x, dtype=torch.float8_e4m3fn, exponents=False, block_rows=1):
    """x [R, D] (any type) -> values of the codes [R, 128 blocks(D)] and scales [blocks(D), blocks of rows], in 64 bits;
    every rounding to f32 that the definition names is made."""
    x = x.to(torch.float64)
    R, D = x.shape
    G = -(-R // block_rows)
    pad = torch.zeros((G * block_rows, blocks(D) * BLOCK), dtype=torch.float64)
    pad[:R, :D] = x
    t = pad.view(G, block_rows, blocks(D), BLOCK)
    amax = torch.where(torch.isfinite(t), t.abs(), torch.zeros_like(t)).amax((1, 3))
    L = LARGEST[dtype]
    if exponents:
        m, e = torch.frexp((amax / L).clamp_min(2.0 ** -126))
        s = torch.ldexp(torch.ones_like(amax), torch.where(m > 0.5, e, e - 1))
    else:
        s = _f32(amax * _f32(torch.tensor(1.0 / L, dtype=torch.float64))).clamp_min(2.0 ** -126)
    v = _f32(t * _f32(1.0 / s)[:, None, :, None])
    return round_codes(v, dtype).view(G * block_rows, -1)[:R], s.t().contiguous()


def values(codes, scales, depth):
    """The matrix [rows, depth] that codes and scales stand for."""
    codes, s = codes.cpu().to(torch.float64), scales.cpu().to(torch.float64).t()
    R = codes.shape[0]
    if s.shape[0] != R:
        s = s.repeat_interleave(BLOCK, 0)[:R]
    return (codes[:, :blocks(depth) * BLOCK].reshape(R, -1, BLOCK) * s[:, :, None]).reshape(R, -1)[:, :depth]


def gate_rows(gate, P, rows_per_gate):
    owner = torch.arange(P) // (rows_per_gate or max(P, 1))
    return gate.to(torch.float64)[owner]


def block_norm(y, h, w_post, w_pre, gate, rows_per_gate, skip, scale, eps):
    """-> u, h', n, 1 / rms(y), 1 / rms(h'), None where there is none."""
    d = lambda t: None if t is None else t.to(torch.float64)  # noqa: E731
    y, h, w_post, w_pre = d(y), d(h), d(w_post), d(w_pre)
    u, r_y = y, torch.ones(len(h), dtype=torch.float64)
    if w_post is not None:
        r_y = 1.0 / torch.sqrt(y.square().mean(1) + eps)
        u = w_post * y * r_y[:, None]
    new = skip * h
    if y is not None:
        g = gate_rows(gate, len(h), rows_per_gate) if gate is not None else 1.0
        new = new + scale * g * u
    n, r_h = None, torch.ones_like(r_y)
    if w_pre is not None:
        r_h = 1.0 / torch.sqrt(new.square().mean(1) + eps)
        n = w_pre * new * r_h[:, None]
    return u, new, n, r_y, r_h


def block_norm_backward(dn, dh, y, h_out, r_y, r_h, w_post, w_pre, gate, rows_per_gate, skip, scale):
    """-> dy, dh_in, dw_post, dw_pre, dgate, None where there is none."""
    d = lambda t: None if t is None else t.to(torch.float64)  # noqa: E731
    dn, dh, y, h, w_post, w_pre = d(dn), d(dh), d(y), d(h_out), d(w_post), d(w_pre)
    t = torch.zeros_like(h) if dh is None else dh
    dw_pre = None if w_pre is None else torch.zeros_like(w_pre)
    if dn is not None:
        hn = h * r_h[:, None]
        a = dn * w_pre
        t = t + r_h[:, None] * (a - hn * (a * hn).mean(1, keepdim=True))
        dw_pre = (dn * hn).sum(0)
    if y is None:
        return None, skip * t, None, dw_pre, None
    yn = y * r_y[:, None] if w_post is not None else y
    w = w_post if w_post is not None else torch.ones(h.shape[1], dtype=torch.float64)
    g = gate_rows(gate, len(h), rows_per_gate) if gate is not None else torch.ones_like(h)
    du = scale * g * t
    b = du * w
    dy = r_y[:, None] * (b - yn * (b * yn).mean(1, keepdim=True)) if w_post is not None else b
    dw_post = (du * yn).sum(0) if w_post is not None else None
    dgate = None
    if gate is not None:
        owner = torch.arange(len(h)) // (rows_per_gate or max(len(h), 1))
        dgate = torch.zeros(gate.shape, dtype=torch.float64).index_add_(0, owner, scale * t * yn * w)
    return dy, skip * t, dw_post, dw_pre, dgate
