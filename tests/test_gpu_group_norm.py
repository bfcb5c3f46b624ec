"""Group norm with an activation and its gradients against plain forms in 64 bits, elementwise, within the roundings there are."""
import pytest

torch = pytest.importorskip("torch")
import more_reference as ref  # noqa: E402
from paper_1905_10830_amd import binding as fmtc  # noqa: E402

pytestmark = pytest.mark.gpu
ACT = {"none": fmtc.ACT_NONE, "relu": fmtc.ACT_RELU, "silu": fmtc.ACT_SILU}
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# samples, rows, channels, groups
SIZES = [(1, 1, 1, 1), (1, 1, 8, 1), (3, 1, 64, 2), (2, 5, 7, 7), (1, 196, 256, 32), (2, 49, 960, 32), (3, 17, 161, 7), (2, 3, 24, 3), (1, 700, 3, 1),
         (5, 64, 64, 32), (1, 3000, 128, 32), (2, 9, 2048, 32), (2, 4, 2049, 1), (1, 3, 8192, 8192), (1, 5, 8192, 1), (1, 2, 5001, 3), (70, 1, 96, 4),
         (300, 2, 40, 5), (2, 1739, 161, 7), (1, 40000, 16, 4), (2, 333, 520, 1), (4, 784, 128, 128), (3, 1025, 64, 1), (1, 2100, 960, 30),
         (1, 5, 15, 5), (3, 40, 27, 9), (2, 300, 33, 11), (1, 3400, 27, 9), (40, 600, 21, 7), (16, 4505, 40, 4), (10, 1364, 1416, 4), (2, 16, 448, 32),
         # slabs of groups that are not multiples of 8, the last of them narrower than 8
         (5, 158, 91, 13), (5, 556, 126, 21), (2, 654, 18, 6), (100, 2154, 25, 5), (1, 7, 245, 35), (20, 1191, 198, 33)]


def _values(samples, rows, C, dtype, seed=0, offset=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((samples * rows, C), generator=g, device="cuda") * torch.exp(0.5 * torch.randn(C, generator=g, device="cuda"))
    return (x + offset * torch.randn(C, generator=g, device="cuda")).to(dtype)


def _params(C, dtype, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return ((1 + 0.3 * torch.randn(C, generator=g, device="cuda")).to(dtype), (0.3 * torch.randn(C, generator=g, device="cuda")).to(dtype))


def _close(got, want, bound):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"off by {float((off / bound).max()):.2f} of the bound"


def _check_stats(stats, want):
    """Both are sums in f64, rounded once (U); r = (variance + eps)^-1/2 has eps as f32 holds it, off by U of it at most, which is
    half that of r where there is no variance: 128 samples of two equal values have it all."""
    for got, w, share in zip(stats.double(), want, (1.01, 1.51)):
        assert bool(((got - w).abs() <= share * ref.U * w.abs() + 1e-12 * want[0].abs().max()).all())


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples, rows, C, groups", SIZES)
def test_forward(samples, rows, C, groups, dtype, act):
    x = _values(samples, rows, C, dtype)
    w, b = _params(C, dtype if (samples + C) % 2 else torch.float32)
    y, stats = fmtc.group_norm(x, groups, w, b, rows_per_sample=rows, act=ACT[act], stats=True)
    want, bound, want_stats = ref.group_norm(x, samples, groups, w, b, act, 1e-5, dtype)
    _close(y, want, bound)
    _check_stats(stats, want_stats)
    plain, none = fmtc.group_norm(x, groups, rows_per_sample=rows, act=ACT[act])
    assert none is None
    _close(plain, *ref.group_norm(x, samples, groups, None, None, act, 1e-5, dtype)[:2])


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples, rows, C, groups", SIZES)
def test_codes(samples, rows, C, groups, dtype, act):
    """The codes of y before it is rounded: within half a code and the error of y, with the scale of the row's largest."""
    x = _values(samples, rows, C, dtype)
    w, b = _params(C, torch.float32)
    q = fmtc.i8_empty(samples * rows, C)
    got, stats = fmtc.group_norm(x, groups, w, b, rows_per_sample=rows, act=ACT[act], out=q, stats=True)
    assert got is q
    want, bound, want_stats = ref.group_norm(x, samples, groups, w, b, act, 1e-5, torch.float32)
    _check_stats(stats, want_stats)
    largest, off = want.abs().amax(1), bound.amax(1)
    assert bool(((q.scales.double() - (largest / 127).clamp_min(2.0 ** -126)).abs() <= off / 127 + 2 * ref.U * largest / 127).all())
    values = q.codes[:, :C].double() * q.scales.double()[:, None]
    # (x (1 / s) and 1 / s are rounded: two half steps of up to 127 codes)
    _close(values, want, bound + q.scales.double()[:, None] * (0.5 + 127 * 3 * ref.U))
    assert not bool(q.codes[:, C:].any())


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples, rows, C, groups", SIZES)
def test_backward(samples, rows, C, groups, dtype, act):
    x = _values(samples, rows, C, dtype)
    dy = _values(samples, rows, C, dtype, 2, offset=0.1)
    w, b = _params(C, dtype if (samples + C) % 2 else torch.float32)
    kw = dict(rows_per_sample=rows, act=ACT[act])
    _, stats = fmtc.group_norm(x, groups, w, b, out=False, stats=True, **kw)
    dx, dw, db = fmtc.group_norm_backward(dy, x, stats, groups, w, b, **kw)
    assert dx.dtype == dtype and dw.dtype == db.dtype == torch.float32
    wants, sizes = ref.group_norm_backward(dy, x, samples, groups, w, b, act, 1e-5, stats)
    # No value passes more than n additions; dz is off by at most 16 roundings of it (the difference to the mean, of x^ and z,
    # and those of the activation's gradient), and where a ReLU's z is within its own error of 0, all of it may be.
    n = rows + C // groups + samples + 64
    _, z_off, _ = ref.group_norm(x, samples, groups, w, b, "none", 1e-5, torch.float32)
    z = ref.group_norm(x, samples, groups, w, b, "none", 1e-5, torch.float32)[0]
    mean, r = (s.double()[:, None, :, None].expand(samples, rows, groups, C // groups).reshape(x.shape) for s in stats)
    xh_off = ref.U * r * (mean.abs() + 2 * (x.double() - mean).abs())
    share = ref.U * (n + 32)
    edge = (z.abs() <= 2 * z_off) if act == "relu" else torch.zeros_like(z, dtype=torch.bool)
    # what of the sums the values at the edge of a ReLU, and the errors of x^ and z, may change
    g = dy.double().abs()
    wd = w.double().abs()
    loose = torch.where(edge, g, torch.zeros_like(g)) + (g * z_off if act == "silu" else 0)
    lost = lambda t: t.view(samples, rows, groups, -1).mean((1, 3), keepdim=True).expand(samples, rows, groups, C // groups).reshape(x.shape)  # noqa: E731
    xh = ((x.double() - mean) * r).abs()
    dx_bound = share * sizes[0] + r * (loose * wd + lost(loose * wd) + xh * lost(loose * wd * xh + g * wd * xh_off) + xh_off * lost(g * wd * xh))
    dx_bound = dx_bound + ref.half_step(dtype) * (wants[0].abs() + dx_bound) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    _close(dx, wants[0], dx_bound)
    _close(dw, wants[1], share * sizes[1] + (loose * (xh + xh_off) + g * xh_off).sum(0) + 1e-30)
    _close(db, wants[2], share * sizes[2] + loose.sum(0) + 1e-30)
    # the errors of all values together are far smaller
    if act != "relu":
        for got, want, limit in zip((dx, dw, db), wants, (ref.half_step(dtype), 0.0, 0.0)):
            assert float((got.double() - want).norm()) <= (limit + 64 * ref.U) * float(want.norm()) + 64 * ref.U * float(sizes[1 if got is dw else 2].norm() if got is not dx else sizes[0].norm())


@pytest.mark.parametrize("act", ref.ACTS)
def test_gradients_are_those_of_the_forward_pass(act):
    """Differences of the forward pass in 64 bits, on the CPU, against the formulas that the kernels are held to."""
    x = _values(2, 6, 12, torch.float32).double().cpu()
    dy = _values(2, 6, 12, torch.float32, 2).double().cpu()
    w, b = (t.double().cpu() for t in _params(12, torch.float32))
    f = lambda x, w, b: float((ref.group_norm(x, 2, 3, w, b, act, 1e-5, torch.float64)[0] * dy).sum())  # noqa: E731
    grads, _ = ref.group_norm_backward(dy, x, 2, 3, w, b, act, 1e-5)
    step = 1e-6
    for which, (at, grad) in enumerate(zip((x, w, b), grads)):
        for i in range(0, at.numel(), 5):
            up, down = ([t.clone() for t in (x, w, b)] for _ in range(2))
            up[which].view(-1)[i] += step
            down[which].view(-1)[i] -= step
            diff = (f(*up) - f(*down)) / (2 * step)
            assert abs(diff - float(grad.view(-1)[i])) <= 1e-6 * (1 + abs(diff))


@pytest.mark.parametrize("samples, rows", [(2, 500), (1, 40000)])
@pytest.mark.parametrize("size", [1e-25, 1e25])
def test_values_whose_squares_leave_f32(size, samples, rows):
    """eps 0: the result is that of the same map at size 1, dx as much smaller as the values are larger"""
    x = _values(samples, rows, 64, torch.float32)
    dy = _values(samples, rows, 64, torch.float32, 2)
    w, b = _params(64, torch.float32)
    kw = dict(rows_per_sample=rows, act=fmtc.ACT_SILU)
    big = x * size
    y, stats = fmtc.group_norm(big, 8, w, b, stats=True, eps=0.0, **kw)
    _close(y, *ref.group_norm(big, samples, 8, w, b, "silu", 0.0, torch.float32)[:2])
    (want, want_w, want_b), (terms, terms_w, terms_b) = ref.group_norm_backward(dy, big, samples, 8, w, b, "silu", 0.0, stats)
    dx, dw, db = fmtc.group_norm_backward(dy, big, stats, 8, w, b, **kw)
    # as many roundings as there are additions, and 48 of the values' own (the difference to the mean, x^, z and the activation)
    share = ref.U * (rows + 8 + samples + 48)
    far = 1 + ((stats[0].abs() * stats[1]).max().double())  # the mean, in deviations: what its rounding is worth
    _close(dx, want, 4 * share * far * terms)
    _close(dw, want_w, 4 * share * far * terms_w)
    _close(db, want_b, 4 * share * far * terms_b)


def test_mean_far_from_zero():
    """A mean of 1000 deviations: the variance is as good as without it, and what is left is the rounding of the mean."""
    x = 1000.0 + _values(2, 500, 64, torch.float32, offset=0.0)
    y, stats = fmtc.group_norm(x, 8, rows_per_sample=500, stats=True)
    want, bound, want_stats = ref.group_norm(x, 2, 8, None, None, "none", 1e-5, torch.float32)
    _close(y, want, bound)
    _check_stats(stats, want_stats)


# in one pass and in two, the last ones in parts; groups of 8, 3, 23 and all channels
FAR = [(2, 196, 64, 8), (3, 50, 27, 9), (7, 1739, 161, 7), (1, 262144, 16, 4), (1, 40000, 40, 1), (2, 3000, 2048, 32)]


@pytest.mark.parametrize("mean, deviation", [(1e4, 1 / 16), (1e5, 1 / 16), (1e6, 1.0), (-3e6, 1.0), (1e30, 1e25)])
@pytest.mark.parametrize("samples, rows, C, groups", FAR)
def test_statistics_wherever_the_mean_is(samples, rows, C, groups, mean, deviation):
    """A mean of 1e5 to 3e6 deviations, without eps: r off by the roundings of f32, as near 0.  (The differences from a group's first
    value are exact in 64 bits; that value is within 6 deviations here, which costs the variance 36 of 2^53.)"""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = mean + deviation * torch.randn((samples * rows, C), generator=g, device="cuda")
    y, stats = fmtc.group_norm(x, groups, rows_per_sample=rows, stats=True, eps=0.0)
    want, bound, want_stats = ref.group_norm(x, samples, groups, None, None, "none", 0.0, torch.float32)
    _close(y, want, bound)
    for got, w in zip(stats.double(), want_stats):  # (rounded once; r in f64 off by far less)
        assert bool(((got - w).abs() <= 1.01 * ref.U * w.abs()).all())
    q = fmtc.i8_empty(samples * rows, C)
    assert torch.equal(fmtc.group_norm(x, groups, rows_per_sample=rows, out=q, stats=True, eps=0.0)[1], stats)
    assert torch.equal(fmtc.group_norm(x, groups, rows_per_sample=rows, out=x, eps=0.0)[0], y)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples, rows, C, groups", FAR)
def test_the_first_value_far_from_the_others(samples, rows, C, groups, dtype):
    """What the sums are taken from lies as far from the mean as one of S D values can: that costs the variance S D of 2^53 at most, and
    the mean half a step of f64 of that value for each addition that it passes.  Of a group that begins with an infinity or a NaN
    all is not a number, but the mean, which is what the sum of its values is."""
    x = _values(samples, rows, C, dtype)
    D = C // groups
    x.view(samples, rows, C)[:, 0, ::D] = 30000.0
    w, b = _params(C, torch.float32)
    y, stats = fmtc.group_norm(x, groups, w, b, rows_per_sample=rows, stats=True)
    want, bound, want_stats = ref.group_norm(x, samples, groups, w, b, "none", 1e-5, dtype)
    _close(y, want, bound)
    added = 2.0 ** -53 * 30000 * (rows + D + 64)
    assert bool(((stats[0].double() - want_stats[0]).abs() <= 1.01 * ref.U * want_stats[0].abs() + added).all())
    assert bool(((stats[1].double() - want_stats[1]).abs() <= 1.51 * ref.U * want_stats[1]).all())
    x.view(samples, rows, C)[-1, 0, 0] = float("inf")
    x.view(samples, rows, C)[0, 0, C - D] = float("nan")
    y, got = fmtc.group_norm(x, groups, w, b, rows_per_sample=rows, stats=True)
    bad = torch.zeros((samples, groups), dtype=torch.bool, device="cuda")
    bad[-1, 0] = bad[0, groups - 1] = True
    assert torch.equal(torch.isnan(got[1]), bad) and torch.equal(got[:, ~bad], stats[:, ~bad])
    if (samples, groups) != (1, 1):
        assert float(got[0, -1, 0]) == float("inf")
    assert torch.equal(torch.isnan(y).view(samples, rows, groups, D).any(3).any(1), bad)


@pytest.mark.parametrize("value", [3.0, 1e5 + 1 / 128, -7e9, 3e4 + 16])
@pytest.mark.parametrize("samples, rows, C, groups", FAR)
def test_maps_of_one_value(samples, rows, C, groups, value):
    """The variance of equal values is 0, not what f64 leaves of the difference of two squares: r is eps^-1/2, rounded (and eps in
    f32: half a step of it, which is half of that of r), y the bias."""
    w, b = _params(C, torch.float32)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.full((samples * rows, C), value, device="cuda").to(dtype)
        y, stats = fmtc.group_norm(x, groups, w, b, rows_per_sample=rows, stats=True)
        assert torch.equal(y, b.to(dtype).expand(x.shape))
        assert bool((stats[0] == x[0, 0].float()).all())
        assert float((stats[1].double() - 1e-5 ** -0.5).abs().max()) <= 1.51 * ref.U * 1e-5 ** -0.5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples, rows, C, groups", FAR)
def test_maps_of_almost_one_value(samples, rows, C, groups, dtype):
    """One value of a group a step away from the others, without eps: a variance of 2^-44 of the mean's square and less.  The last value
    of a group, and (second sample, or all groups but the first) its first one."""
    base = torch.full((1,), 200.0, device="cuda").to(dtype)
    step = torch.nextafter(base.cpu(), torch.full((1,), 1e4, dtype=dtype)).to("cuda")
    x = base.expand(samples * rows, C).clone()
    v = x.view(samples, rows, groups, C // groups)
    v[0, -1, 0, -1] = step
    v[0, 0, 1:, 0] = step
    v[1:, 0, :, 0] = step
    y, stats = fmtc.group_norm(x, groups, rows_per_sample=rows, stats=True, eps=0.0)
    n, off = rows * C // groups, float(step) - float(base)
    r = 1.0 / (off * (1.0 / n * (1.0 - 1.0 / n)) ** 0.5)  # n - 1 equal values and one: (n - 1) / n^2 off^2
    assert bool(((stats[1].double() - r).abs() <= 1.01 * ref.U * r).all())
    assert bool(((stats[0].double() - (float(base) + off / n)).abs() <= 1.01 * ref.U * float(step)).all())
    want, bound, _ = ref.group_norm(x, samples, groups, None, None, "none", 0.0, dtype)
    _close(y, want, bound)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_strides(dtype):
    samples, rows, C, groups = 3, 50, 96, 8
    wide = _values(samples, rows, C + 11, dtype)
    x = wide[:, 5:5 + C]
    keep = wide.clone()
    w, b = _params(C, dtype)
    kw = dict(rows_per_sample=rows, act=fmtc.ACT_SILU)
    want, stats = fmtc.group_norm(x.contiguous(), groups, w, b, stats=True, **kw)
    store = torch.full((samples * rows, C + 6), 3.0, dtype=dtype, device="cuda")
    assert torch.equal(fmtc.group_norm(x, groups, w, b, out=store[:, 1:1 + C], **kw)[0], want)
    assert bool((store[:, 0] == 3.0).all()) and bool((store[:, 1 + C:] == 3.0).all())
    dy = _values(samples, rows, C, dtype, 3)
    grads = fmtc.group_norm_backward(dy, x.contiguous(), stats, groups, w, b, **kw)
    dy_wide = torch.full((samples * rows, C + 3), 2.0, dtype=dtype, device="cuda")
    dy_wide[:, 2:2 + C] = dy
    got = fmtc.group_norm_backward(dy_wide[:, 2:2 + C], x, stats, groups, w, b, dx=dy_wide[:, 2:2 + C], **kw)
    assert all(torch.equal(a, c) for a, c in zip(got, grads))
    assert bool((dy_wide[:, :2] == 2.0).all()) and bool((dy_wide[:, 2 + C:] == 2.0).all())
    assert torch.equal(fmtc.group_norm(x, groups, w, b, out=x, **kw)[0], want)
    assert torch.equal(wide[:, :5], keep[:, :5]) and torch.equal(wide[:, 5 + C:], keep[:, 5 + C:])
    x.copy_(keep[:, 5:5 + C])
    assert torch.equal(fmtc.group_norm_backward(dy, x, stats, groups, w, b, dx=x, **kw)[0], grads[0])


def test_in_place_of_rows_of_an_odd_length():
    x = _values(2, 300, 161, torch.bfloat16)
    want, _ = fmtc.group_norm(x, 7, rows_per_sample=300, act=fmtc.ACT_RELU)
    assert torch.equal(fmtc.group_norm(x, 7, rows_per_sample=300, act=fmtc.ACT_RELU, out=x)[0], want)


@pytest.mark.parametrize("weight, bias", [(True, False), (False, True)])
def test_one_of_weight_and_bias(weight, bias):
    x, dy = _values(2, 40, 48, torch.float16), _values(2, 40, 48, torch.float16, 1)
    w, b = (t if there else None for t, there in zip(_params(48, torch.float16), (weight, bias)))
    y, stats = fmtc.group_norm(x, 6, w, b, rows_per_sample=40, stats=True)
    _close(y, *ref.group_norm(x, 2, 6, w, b, "none", 1e-5, torch.float16)[:2])
    dx, dw, db = fmtc.group_norm_backward(dy, x, stats, 6, w, b, rows_per_sample=40)
    assert (dw is not None, db is not None) == (weight, bias)
    (want, want_w, want_b), _ = ref.group_norm_backward(dy, x, 2, 6, w, b, "none", 1e-5, stats)
    assert float((dx.double() - want).norm()) <= (2.0 ** -11 + 64 * ref.U) * float(want.norm())
    for got, full in ((dw, want_w), (db, want_b)):
        assert got is None or float((got.double() - full).norm()) <= 128 * ref.U * float(full.norm())
    only = fmtc.group_norm_backward(dy, x, stats, 6, w, b, rows_per_sample=40, dx=False)
    assert only[0] is None and all((a is None) == (c is None) and (a is None or torch.equal(a, c)) for a, c in zip(only[1:], (dw, db)))


# in one pass and in two, with sums of parts in every number
MANY = [(1000, 1, 64, 8), (2049, 3, 64, 8), (5000, 1, 40, 5), (70000, 1, 16, 2), (3000, 1, 264, 33), (9, 30000, 8, 1), (2100, 1, 4104, 1), (2300, 400, 64, 1)]


@pytest.mark.parametrize("dx", [None, False])
@pytest.mark.parametrize("samples, rows, C, groups", MANY)
def test_parameter_gradients_of_many_samples(samples, rows, C, groups, dx):
    """Gradients of 4 / 3 everywhere: f32 sums one after the other lose the same part of a step each time.  Within a sample's part there
    are no more additions than rows, the parts are added up in f64; two roundings to f32 at the end."""
    x = _values(samples, rows, C, torch.float32)
    dy = torch.full_like(x, 4 / 3)
    w, b = _params(C, torch.float32)
    _, stats = fmtc.group_norm(x, groups, w, b, rows_per_sample=rows, out=False, stats=True)
    _, dw, db = fmtc.group_norm_backward(dy, x, stats, groups, w, b, rows_per_sample=rows, dx=dx)
    (_, want_w, want_b), (_, size_w, size_b) = ref.group_norm_backward(dy, x, samples, groups, w, b, "none", 1e-5, stats)
    added = min(rows, 1500)  # (a sample of more rows is cut in parts, each of its threads' sums is a part of that)
    _close(db, want_b, ref.U * (added + 1.02) * size_b)
    _close(dw, want_w, ref.U * (added + 1.02 + 3) * size_w)  # (and each dz x^: the difference, the product with r, and with dz)


# workgroups of every size: 64, 128 and 256 threads for samples of few rows
SMALL = [(9000, 1, 64, 8), (9000, 7, 64, 8), (9001, 16, 64, 8), (8200, 3, 27, 9), (8193, 1, 520, 5), (8200, 1, 1000, 125), (9000, 2, 7, 7), (20000, 1, 2, 1),
         (8200, 60, 15, 5), (8200, 1, 1032, 1), (2100, 1, 520, 65), (9000, 1, 91, 13)]


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("samples, rows, C, groups", SMALL)
def test_many_small_samples(samples, rows, C, groups, dtype, act):
    test_forward(samples, rows, C, groups, dtype, act)
    test_codes(samples, rows, C, groups, dtype, act)
    test_backward(samples, rows, C, groups, dtype, act)


# more samples than a launch takes, by a few; more than HIP's 2^32 threads would take with a workgroup each
SEVERAL = [(2 * 131072 + 3, 1, 64, 8), (2048 + 5, 2, 8184, 8184), (2043 + 3, 2, 4104, 3), (1024 + 1, 3, 8192, 1), ((1 << 24) + 5, 1, 8, 2)]


@pytest.mark.parametrize("samples, rows, C, groups", SEVERAL)
def test_samples_of_several_launches(samples, rows, C, groups):
    x = _values(samples, rows, C, torch.float32)
    w, b = _params(C, torch.float32)
    kw = dict(rows_per_sample=rows)
    y, stats = fmtc.group_norm(x, groups, w, b, stats=True, **kw)
    want, bound, want_stats = ref.group_norm(x, samples, groups, w, b, "none", 1e-5, torch.float32)
    _close(y, want, bound)
    _check_stats(stats, want_stats)
    q = fmtc.i8_empty(samples * rows, C)
    fmtc.group_norm(x, groups, w, b, out=q, **kw)
    off = bound + q.scales.double()[:, None] * (0.5 + 127 * 3 * ref.U)
    _close(q.codes[:, :C].double() * q.scales.double()[:, None], want, off)
    del want, bound, off, q
    dy = torch.full_like(x, 4 / 3)
    dy[::2] = -0.3
    (want, want_w, want_b), (terms, size_w, size_b) = ref.group_norm_backward(dy, x, samples, groups, w, b, "none", 1e-5, stats)
    far = 1 + ((stats[0].abs() * stats[1]).max().double())  # the mean, in deviations: what its rounding is worth
    for dx in (None, False):
        got, dw, db = fmtc.group_norm_backward(dy, x, stats, groups, w, b, dx=dx, **kw)
        if dx is None:
            _close(got, want, 4 * ref.U * (rows + C // groups + 64) * far * terms)
        _close(db, want_b, ref.U * (rows + 1.02) * size_b)
        _close(dw, want_w, ref.U * (rows + 1.02 + 3) * size_w)


def test_no_rows():
    x = torch.empty((0, 48), dtype=torch.bfloat16, device="cuda")
    w, b = _params(48, torch.float32)
    y, stats = fmtc.group_norm(x, 6, w, b, stats=True)
    assert y.shape == (0, 48) and stats.shape == (2, 0, 6)
    dx, dw, db = fmtc.group_norm_backward(x, x, stats, 6, w, b)
    assert dx.shape == (0, 48) and not bool(dw.any()) and not bool(db.any()) and dw.shape == db.shape == (48,)
    assert fmtc.group_norm(x, 6, w, b, out=fmtc.i8_empty(0, 48))[0].rows == 0


def test_a_value_that_is_not_a_number_stays_in_its_group():
    x = _values(2, 30, 64, torch.bfloat16)
    clean = x.clone()
    x[35, 9] = float("nan")  # sample 1, group 1 of 8
    kw = dict(rows_per_sample=30, act=fmtc.ACT_RELU)
    y, stats = fmtc.group_norm(x, 8, stats=True, **kw)
    want, want_stats = fmtc.group_norm(clean, 8, stats=True, **kw)
    bad = torch.zeros((60, 64), dtype=torch.bool, device="cuda")
    bad[30:, 8:16] = True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], want[~bad])
    assert torch.equal(torch.isnan(stats), torch.isnan(torch.where(torch.tensor([[False] * 8, [False, True] + [False] * 6], device="cuda"), float("nan"), want_stats)))


def test_constant_maps():
    """a variance of 0: eps alone, and of all 0 exactly the bias"""
    x = torch.full((20, 16), 3.0, dtype=torch.float32, device="cuda")
    w, b = _params(16, torch.float32)
    y, stats = fmtc.group_norm(x, 4, w, b, stats=True)
    assert torch.equal(y, b.expand(20, 16)) and bool((stats[0] == 3.0).all())
    assert float((stats[1] - 1e-5 ** -0.5).abs().max()) <= 2 * ref.U * 1e-5 ** -0.5


@pytest.mark.parametrize("samples, rows, C, groups", [(2, 1739, 161, 7), (32, 196, 256, 32), (1, 40000, 16, 4)])
def test_the_same_numbers_in_every_run(samples, rows, C, groups):
    x, dy = _values(samples, rows, C, torch.bfloat16), _values(samples, rows, C, torch.bfloat16, 1)
    w, b = _params(C, torch.float32)
    kw = dict(rows_per_sample=rows, act=fmtc.ACT_SILU)

    def run():
        y, stats = fmtc.group_norm(x, groups, w, b, stats=True, **kw)
        return y, stats, *fmtc.group_norm_backward(dy, x, stats, groups, w, b, **kw)
    first = run()
    for _ in range(4):
        assert all(torch.equal(a, c) for a, c in zip(run(), first))
