"""Norms, gate and residual between two blocks (fmtc_block_norm) and their gradients on the GPU, against plain 64-bit
ones."""
import pytest

torch = pytest.importorskip("torch")
import f8_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}  # of 1, 8 / 11 / 24 significant bits
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -140}
EPS = 1e-6
# every width of the kernels' rows, and odd ones beside it
WIDTHS = [1, 8, 100, 128, 129, 512, 577, 1024, 1025, 2048, 4095, 4096, 8192, 9001, 16384]


@pytest.fixture(scope="module")
def fmtc():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_10830_amd import binding

    binding.load_library()
    return binding


class Case:
    def __init__(self, P, C, dtype=torch.bfloat16, weights=torch.float32, rows_per_gate=0, skip=1.0, scale=1.0, seed=0, gate=True,
                 y=True, post=True, pre=True):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.P, self.C, self.dtype = P, C, dtype
        self.y = (3 * r(P, C)).to(dtype) if y else None
        self.h = (r(P, C) * torch.exp(r(P, 1))).to(dtype)
        self.w_post = (1 + 0.3 * r(C)).to(weights) if post and y else None
        self.w_pre = (1 + 0.3 * r(C)).to(weights) if pre else None
        G = -(-P // rows_per_gate) if rows_per_gate else 1
        self.gate = r(G, C).to(weights) if gate and y else None
        self.more = dict(rows_per_gate=rows_per_gate, skip=skip, scale=scale)
        self.dn = (1e-2 * r(P, C)).to(dtype)
        self.dh = (1e-2 * r(P, C)).to(dtype)

    def on(self, t):
        return None if t is None else t.cuda()

    def forward(self, fmtc, **more):
        on = self.on
        return fmtc.block_norm(on(self.y), on(self.h), on(self.w_post), on(self.w_pre), gate=on(self.gate), eps=EPS, **self.more, **more)

    def want(self):
        return ref.block_norm(self.y, self.h, self.w_post, self.w_pre, self.gate, self.more["rows_per_gate"], self.more["skip"],
                              self.more["scale"], EPS)


def _near(got, want, rel, more=0.0, what=""):
    off = (got.cpu().to(torch.float64) - want).abs()
    limit = rel * want.abs() + more
    assert (off <= limit).all(), f"{what}: {float((off / limit).max())} of the limit"


def _check_forward(fmtc, c):
    h, n, stats = c.forward(fmtc, stats=True)
    u, wh, wn, r_y, r_h = c.want()
    half, tiny = HALF_ULP[c.dtype], TINY[c.dtype]
    # a sum of C squares in f32 by lanes of up to 16 and a tree: under 32 roundings, halved by the root, and a few more
    f32 = 24 * 2.0 ** -24
    part = (c.more["scale"] * ref.gate_rows(c.gate, c.P, c.more["rows_per_gate"]) * u).abs() if c.gate is not None else 0 if u is None else (c.more["scale"] * u).abs()
    own = f32 * (part + (c.more["skip"] * c.h.double()).abs())
    _near(h, wh, 1.01 * half, own + tiny, "h'")
    if c.y is not None and c.w_post is not None:
        _near(stats[0], r_y, f32, 0, "1 / rms(y)")
    if n is None:
        return
    # what the parts of h' lost in f32 shows in its norm by its size against the whole row's
    lost = own * r_h[:, None] * c.w_pre.double().abs()
    tilt = (own.square().sum(1).sqrt() / wh.square().sum(1).sqrt().clamp_min(1e-30))[:, None]
    _near(stats[1], r_h, f32 + tilt[:, 0], 0, "1 / rms(h')")
    _near(n, wn, 1.01 * half + f32 + tilt, lost + tiny, "n")


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward_of_every_width(fmtc, C, dtype):
    _check_forward(fmtc, Case(5, C, dtype, rows_per_gate=2, skip=0.9, scale=0.5, seed=C))


@pytest.mark.parametrize("weights", ["own", "f32"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P, rows_per_gate", [(1, 1), (7, 0), (33, 1), (33, 5), (40, 40), (40, 64), (3000, 1000)])
def test_forward_of_every_gate(fmtc, P, rows_per_gate, dtype, weights):
    _check_forward(fmtc, Case(P, 200, dtype, dtype if weights == "own" else torch.float32, rows_per_gate, seed=P))


PARTS = [dict(gate=False), dict(post=False), dict(pre=False), dict(y=False), dict(gate=False, post=False), dict(post=False, pre=False)]


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("C", [96, 1000, 4096])
def test_forward_without_some_of_its_parts(fmtc, parts, C):
    _check_forward(fmtc, Case(9, C, rows_per_gate=4, scale=0.7, seed=5, **parts))


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("exponents", [False, True])
@pytest.mark.parametrize("e5m2", [False, True])
def test_codes_are_those_of_the_quantizer(fmtc, C, exponents, e5m2):
    """In f32 the row that is stored and the row that is quantized are the same one, so the codes have to be equal."""
    kinds = dict(fmt=fmtc.E5M2 if e5m2 else fmtc.E4M3, scales=fmtc.SCALE_E8M0 if exponents else fmtc.SCALE_F32)
    c = Case(6, C, torch.float32, rows_per_gate=3, seed=C + 1)
    q = fmtc.f8_empty(6, C, **kinds)
    h, n, _ = c.forward(fmtc)
    h2, _, _ = c.forward(fmtc, n_out=q)
    want, _ = fmtc.f8_quantize(n, **kinds)
    assert torch.equal(h, h2) and torch.equal(q.scales, want.scales)
    assert torch.equal(q.codes.view(torch.uint8), want.codes.view(torch.uint8))


def test_rows_of_zeros_and_of_what_is_not_finite(fmtc):
    c = Case(6, 300, torch.float32, rows_per_gate=1, seed=3)
    c.y[0] = 0.0
    c.h[0] = 0.0
    c.y[1] = 0.0
    c.y[2, 5] = float("nan")
    c.h[3, 7] = float("inf")
    h, n, stats = c.forward(fmtc, stats=True)
    h, n, stats = h.cpu(), n.cpu(), stats.cpu()
    assert not h[0].any() and not n[0].any()
    assert torch.allclose(stats[:, 0], torch.full((2,), EPS ** -0.5), rtol=1e-5)
    assert torch.equal(h[1], c.h[1])
    assert torch.isnan(h[2]).all() and torch.isnan(n[2]).all()
    assert torch.isinf(h[3, 7]) and torch.isnan(n[3, 7]) and not torch.isnan(h[3]).any()
    for row in (4, 5):
        assert torch.isfinite(n[row]).all()


def test_in_place_strides_streams_and_no_rows(fmtc):
    c = Case(20, 1000, rows_per_gate=7, seed=8)
    h, n, stats = c.forward(fmtc, stats=True)
    wide_h = torch.zeros((20, 1027), dtype=c.dtype, device="cuda")
    wide_n = torch.zeros((20, 1033), dtype=c.dtype, device="cuda")
    view = wide_h[:, 3:1003]
    view.copy_(c.h.cuda())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fmtc.block_norm(c.y.cuda(), view, c.w_post.cuda(), c.w_pre.cuda(), gate=c.gate.cuda(), eps=EPS, h_out=view,
                        n_out=wide_n[:, 1:1001], **c.more)
    side.synchronize()
    assert torch.equal(view, h) and torch.equal(wide_n[:, 1:1001], n)
    assert not wide_h[:, :3].any() and not wide_h[:, 1003:].any() and not wide_n[:, 0].any() and not wide_n[:, 1001:].any()
    only, none, _ = c.forward(fmtc, h_out=False)
    assert only is None and torch.equal(none, n)
    e = Case(0, 64, gate=False)
    h, n, _ = e.forward(fmtc)
    assert h.shape == (0, 64)


def _check_backward(fmtc, c, dn=True, dh=True):
    on = c.on
    h, _, stats = c.forward(fmtc, stats=True)
    dn, dh = c.dn if dn and c.w_pre is not None else None, c.dh if dh else None
    got = fmtc.block_norm_backward(on(dn), on(dh), on(c.y), h, stats, on(c.w_post), on(c.w_pre), gate=on(c.gate), **c.more)
    hc, s = h.cpu(), stats.cpu().double()
    want = ref.block_norm_backward(dn, dh, c.y, hc, s[0], s[1], c.w_post, c.w_pre, c.gate, **c.more)
    half, tiny = HALF_ULP[c.dtype], TINY[c.dtype]
    f32 = 2.0 ** -24
    # sizes of what is added up: rows' sums of C products each, in lanes of up to 16 and trees, scaled back by the row
    size = lambda t: t.double().abs() if t is not None else 0.0  # noqa: E731
    hn = (hc.double() * s[1][:, None]).abs() if dn is not None else 0.0
    a = size(dn) * size(c.w_pre) if dn is not None else 0.0
    t = size(dh) + (s[1][:, None] * (a + hn * (a * hn).mean(1, keepdim=True)) if dn is not None else torch.zeros_like(hc.double()))
    _near(got[1], want[1], 1.01 * half, 64 * f32 * abs(c.more["skip"]) * t + tiny, "dh")
    if dn is not None:
        _near(got[3], want[3], 0, (16 + c.P / 16) * f32 * (size(dn) * hn).sum(0) + 1e-30, "dw_pre")
    if c.y is None:
        assert got[0] is None
        return
    yn = (c.y.double() * s[0][:, None]).abs() if c.w_post is not None else c.y.double().abs()
    w = size(c.w_post) if c.w_post is not None else 1.0
    g = size(ref.gate_rows(c.gate, c.P, c.more["rows_per_gate"])) if c.gate is not None else 1.0
    b = c.more["scale"] * g * w * t
    dy = s[0][:, None] * (b + yn * (b * yn).mean(1, keepdim=True)) if c.w_post is not None else b
    _near(got[0], want[0], 1.01 * half, 128 * f32 * dy + tiny, "dy")
    if c.w_post is not None:
        _near(got[2], want[2], 0, (96 + c.P / 16) * f32 * (c.more["scale"] * g * t * yn).sum(0) + 1e-30, "dw_post")
    if c.gate is not None:
        owner = torch.arange(c.P) // (c.more["rows_per_gate"] or c.P)
        most = torch.zeros(c.gate.shape, dtype=torch.float64).index_add_(0, owner, c.more["scale"] * t * yn * w)
        assert got[4].shape == c.gate.shape
        _near(got[4], want[4], 0, (96 + c.P / 16) * f32 * most + 1e-30, "dgate")


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_every_width(fmtc, C, dtype):
    _check_backward(fmtc, Case(11, C, dtype, rows_per_gate=4, skip=0.9, scale=0.5, seed=C))


@pytest.mark.parametrize("weights", ["own", "f32"])
@pytest.mark.parametrize("P, C, rows_per_gate", [(1, 64, 1), (7, 64, 0), (33, 64, 1), (500, 130, 3), (500, 130, 5), (40, 1500, 64),
                                                 (3000, 600, 1000), (2999, 600, 1000), (1010, 2000, 1000), (9000, 40, 4000)])
def test_gradients_of_every_gate(fmtc, P, C, rows_per_gate, weights):
    _check_backward(fmtc, Case(P, C, torch.bfloat16, torch.bfloat16 if weights == "own" else torch.float32, rows_per_gate, scale=0.5, seed=P))


@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("C", [96, 1000, 4096])
def test_gradients_without_some_parts(fmtc, parts, C):
    _check_backward(fmtc, Case(21, C, rows_per_gate=4, scale=0.7, seed=5, **parts))
    if parts.get("pre", True):
        _check_backward(fmtc, Case(21, C, rows_per_gate=4, scale=0.7, seed=6, **parts), dh=False)
        _check_backward(fmtc, Case(21, C, rows_per_gate=4, scale=0.7, seed=7, **parts), dn=False)


def test_gradients_of_no_rows(fmtc):
    c = Case(0, 100, gate=False)
    h, _, stats = c.forward(fmtc, stats=True)
    on = c.on
    got = fmtc.block_norm_backward(on(c.dn), on(c.dh), on(c.y), h, stats, on(c.w_post), on(c.w_pre))
    assert got[0].shape == (0, 100) and not got[2].any() and not got[3].any()


@pytest.mark.parametrize("which", ["y", "h", "w_post", "w_pre", "gate"])
def test_gradients_equal_differences(fmtc, which):
    """A step of 1/64 both ways along a random direction, in f32: the loss' third derivative along it is of the order of its
    first, so the difference is off by about (1/64)^2 / 6 = 4e-5 of that, and by 1e-6 * 64 from f32 sums."""
    c = Case(12, 200, torch.float32, rows_per_gate=5, skip=0.9, scale=0.5, seed=11)
    c.h = torch.randn((12, 200), generator=torch.Generator().manual_seed(1))
    at = getattr(c, which)
    direction = torch.randn(at.shape, generator=torch.Generator().manual_seed(2))

    def loss(step):
        setattr(c, which, at + step * direction)
        h, n, _ = c.forward(fmtc)
        return float((c.dn.double() * n.cpu().double()).sum() + (c.dh.double() * h.cpu().double()).sum())

    slope = (loss(1 / 64) - loss(-1 / 64)) * 32
    setattr(c, which, at)
    h, _, stats = c.forward(fmtc, stats=True)
    on = c.on
    got = fmtc.block_norm_backward(on(c.dn), on(c.dh), on(c.y), h, stats, on(c.w_post), on(c.w_pre), gate=on(c.gate), **c.more)
    grad = got[["y", "h", "w_post", "w_pre", "gate"].index(which)].cpu().double()
    exact = float((grad * direction.double()).sum())
    assert abs(slope - exact) <= 2e-3 * float((grad.norm() * direction.double().norm()) / grad.numel() ** 0.5)


def test_gradients_give_the_same_bits_every_time(fmtc):
    for C in (64, 600, 4096):
        c = Case(700, C, rows_per_gate=300, seed=C)
        h, _, stats = c.forward(fmtc, stats=True)
        on = c.on
        runs = [fmtc.block_norm_backward(on(c.dn), on(c.dh), on(c.y), h, stats, on(c.w_post), on(c.w_pre), gate=on(c.gate), **c.more)
                for _ in range(3)]
        assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


def test_rows_far_apart(fmtc):
    """Offsets past 2^32 bytes."""
    step = (1 << 30) + 8
    room = torch.zeros(4 * step + 512, dtype=torch.bfloat16, device="cuda")
    c = Case(5, 200, rows_per_gate=2, seed=12)
    h, n, stats = c.forward(fmtc, stats=True)
    far = room.as_strided((5, 200), (step, 1))
    far.copy_(c.h.cuda())
    on = c.on
    fmtc.block_norm(on(c.y), far, on(c.w_post), on(c.w_pre), gate=on(c.gate), eps=EPS, h_out=far, **c.more)
    assert torch.equal(far, h)
    near = fmtc.block_norm_backward(on(c.dn), on(c.dh), on(c.y), h, stats, on(c.w_post), on(c.w_pre), gate=on(c.gate), **c.more)
    again = fmtc.block_norm_backward(on(c.dn), on(c.dh), on(c.y), far, stats, on(c.w_post), on(c.w_pre), gate=on(c.gate), **c.more)
    assert all(torch.equal(a, b) for a, b in zip(near, again))
    del room, far
    torch.cuda.empty_cache()


def test_refusals_of_the_binding(fmtc):
    c = Case(6, 64, rows_per_gate=2, seed=13)
    on = c.on
    y, h, w1, w2, gate = map(on, (c.y, c.h, c.w_post, c.w_pre, c.gate))
    with pytest.raises(fmtc.FmtcError, match="eps"):
        fmtc.block_norm(y, h, w1, w2, eps=-1.0)
    with pytest.raises(fmtc.FmtcError, match="w_post and gate need y"):
        fmtc.block_norm(None, h, w1, w2)
    with pytest.raises(fmtc.FmtcError, match="n needs w_pre"):
        fmtc.block_norm(y, h, w1, None, n_out=torch.empty_like(h))
    with pytest.raises(fmtc.FmtcError, match="n_codes"):
        fmtc.block_norm(y, h, w1, w2, n_out=fmtc.f8_empty(6, 64, block_rows=128))
    for bad in (lambda: fmtc.block_norm(y.float(), h, w1, w2), lambda: fmtc.block_norm(y[:5], h, w1, w2),
                lambda: fmtc.block_norm(y, h, w1[:63], w2), lambda: fmtc.block_norm(y, h, w1, w2.to(torch.bfloat16)),
                lambda: fmtc.block_norm(y, h, w1, w2, gate=gate, rows_per_gate=3),
                lambda: fmtc.block_norm(y, h, w1, w2, stats=torch.empty((2, 5), device="cuda")),
                lambda: fmtc.block_norm(y, h.t(), w1, w2), lambda: fmtc.block_norm(y, h.cpu(), w1, w2)):
        with pytest.raises(ValueError):
            bad()
