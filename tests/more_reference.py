"""Plain implementations of the products in 8-bit integers, the group norm and the clipped gradients, in 64 bits, with bounds
on what 32-bit steps may add (u: half a step of f32; every rounding is off by at most that share of its result)."""
import torch

U = 2.0 ** -24
BLOCK = 128


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def codes(x):
    """The codes (int8, [rows, cols]) and scales of rows, step by step in f32 as they are defined."""
    x = x.float()
    bits = x.abs().amax(1)
    finite = torch.isfinite(x).all(1)
    s = (bits * torch.tensor(1 / 127, dtype=torch.float32)).clamp_min(2.0 ** -126)
    q = torch.round(x * (1.0 / s)[:, None])
    q = torch.where(finite[:, None], q, torch.zeros_like(q)).to(torch.int8)
    return q, torch.where(finite, s, torch.full_like(s, float("nan")))


def pad(q):
    return torch.nn.functional.pad(q, (0, -q.shape[1] % BLOCK))


def product(qa, sa, qb, sb, bias, dtype):
    """-> exact values, bound on the error of results in dtype"""
    y = (qa.double() @ qb.double().t()) * sa.double()[:, None] * sb.double()
    bound = 3 * U * y.abs()                 # the sum to f32, two factors
    if bias is not None:
        y = y + bias.double()
        bound = bound + U * (y.abs() + bound)
    return y, bound * (1 + 8 * U) + half_step(dtype) * (y.abs() + bound) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


ACTS = ("none", "relu", "silu")


def _act(z, act):
    return z if act == "none" else torch.where(z < 0, torch.zeros_like(z), z) if act == "relu" else z * torch.sigmoid(z)


def _parts(x, samples, groups):
    P, C = x.shape
    return x.double().view(samples, -1, groups, C // groups)


def _affine(weight, bias, groups, like):
    C = like.shape[1]
    w = torch.ones(C, dtype=torch.float64, device=like.device) if weight is None else weight.double()
    b = torch.zeros(C, dtype=torch.float64, device=like.device) if bias is None else bias.double()
    return w.view(1, 1, groups, -1), b.view(1, 1, groups, -1)


def group_norm(x, samples, groups, weight, bias, act, eps, dtype):
    """-> y, bound, stats [2, samples, groups]"""
    w, b = _affine(weight, bias, groups, x)
    v = _parts(x, samples, groups)
    mean = v.mean((1, 3), keepdim=True)
    r = 1 / torch.sqrt((v - mean).square().mean((1, 3), keepdim=True) + eps)
    z = (v - mean) * r * w + b
    # the mean rounded, the difference, r rounded, r w, the product with the sum
    bound = U * (mean.abs() * (r * w).abs() + 3 * ((v - mean) * r * w).abs() + z.abs())
    y = _act(z, act)
    # |silu'| < 1.1; silu itself: z log2 e rounded before 2^z (2 |z| u e / (1 + e) <= u), then 2^z, sum, reciprocal, product
    bound = 1.1 * bound + (8 * U * y.abs() if act == "silu" else 0)
    bound = bound * (1 + 16 * U) + half_step(dtype) * (y.abs() + bound) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    return y.view(x.shape), bound.view(x.shape), torch.stack([mean.view(samples, groups), r.view(samples, groups)])


def group_norm_backward(dy, x, samples, groups, weight, bias, act, eps, stats=None):
    """-> dx, dweight, dbias by the formulas, with what bounds their errors: (|terms| of dx, sums of |terms| of the others)"""
    w, b = _affine(weight, bias, groups, x)
    v, g = _parts(x, samples, groups), _parts(dy, samples, groups)
    if stats is None:
        mean = v.mean((1, 3), keepdim=True)
        r = 1 / torch.sqrt((v - mean).square().mean((1, 3), keepdim=True) + eps)
    else:
        mean, r = (s.double()[:, None, :, None] for s in stats)
    xh = (v - mean) * r
    z = xh * w + b
    if act == "relu":
        g = torch.where(z > 0, g, torch.zeros_like(g))
    elif act == "silu":
        p = torch.sigmoid(z)
        g = g * (p + z * p * torch.sigmoid(-z))
    a = g * w
    A, B = a.mean((1, 3), keepdim=True), (a * xh).mean((1, 3), keepdim=True)
    dx = r * (a - A - xh * B)
    terms = r * (a.abs() + a.abs().mean((1, 3), keepdim=True) + xh.abs() * (a * xh).abs().mean((1, 3), keepdim=True))
    flat = lambda t: t.sum((0, 1)).reshape(-1)  # noqa: E731
    return ((dx.view(x.shape), flat(g * xh), flat(g)),
            (terms.view(x.shape), flat((g * xh).abs()), flat(g.abs())))


def clip(tensors, max_norm, scale, eps):
    """-> norm, factor (in 64 bits)"""
    total = sum(float(t.double().square().sum()) for t in tensors)
    norm = scale * total ** 0.5
    return norm, scale * min(1.0, max_norm / (norm + eps))
