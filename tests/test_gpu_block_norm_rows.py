"""Norms and their gradients where a workgroup walks over several rows: rows in turn and consecutive ones, the row that is
loaded ahead, gates that change on the way, strips of whole gate rows, the last pass with rows that do not exist; codes of
streams in every type."""
import pytest

torch = pytest.importorskip("torch")
import f8_reference as ref  # noqa: E402
from test_gpu_block_norm import EPS, TYPES, Case, _check_backward, _check_forward, fmtc  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# rows and channels: 3 passes and more of all the workgroups of a launch (1024 of 256 lanes, 512 of 512, 256 of 1024; a row takes
# 16, 64, 128, 256, 512 or 1024 lanes), the last one not full
MANY = [(2 * 16384 + 50, 40), (2 * 16384 + 1, 100), (9001, 300), (8193, 512), (5001, 1000), (2500, 2000), (1300, 4096), (1301, 4095),
        (700, 8192), (701, 8191), (600, 9001), (601, 16384)]


@pytest.mark.parametrize("P, C", MANY)
@pytest.mark.parametrize("rows_per_gate", [None, 0, 7, 300])
def test_forward_of_many_rows(fmtc, P, C, rows_per_gate):  # noqa: F811
    _check_forward(fmtc, Case(P, C, rows_per_gate=rows_per_gate or 0, gate=rows_per_gate is not None, skip=0.9, scale=0.5, seed=P))


@pytest.mark.parametrize("P, C", [(9001, 300), (1300, 4096), (701, 8191), (600, 16384)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_forward_of_many_rows_in_other_types(fmtc, P, C, dtype):  # noqa: F811
    _check_forward(fmtc, Case(P, C, dtype, dtype, rows_per_gate=90, seed=C))
    _check_forward(fmtc, Case(P, C, dtype, gate=False, post=False, seed=C))
    _check_forward(fmtc, Case(P, C, dtype, y=False, seed=C))


@pytest.mark.parametrize("P, C", MANY)
@pytest.mark.parametrize("rows_per_gate", [0, 7])
def test_many_rows_in_place(fmtc, P, C, rows_per_gate):  # noqa: F811
    c = Case(P, C, rows_per_gate=rows_per_gate, seed=C)
    on = c.on
    h, n, stats = c.forward(fmtc, stats=True)
    own = on(c.h)
    _, n2, stats2 = fmtc.block_norm(on(c.y), own, on(c.w_post), on(c.w_pre), gate=on(c.gate), eps=EPS, h_out=own, stats=True, **c.more)
    assert torch.equal(own, h) and torch.equal(n2, n) and torch.equal(stats2, stats)
    back = lambda **more: fmtc.block_norm_backward(on(c.dn), dh, on(c.y), h, stats, on(c.w_post), on(c.w_pre), gate=on(c.gate), **c.more, **more)  # noqa: E731
    dh = on(c.dh)
    want = back()
    got = back(dh_in=dh)
    assert got[1] is dh and all(torch.equal(a, b) for a, b in zip(got, want, strict=True))


@pytest.mark.parametrize("P, C", MANY)
@pytest.mark.parametrize("e5m2, exponents", [(False, False), (False, True), (True, False)])
def test_codes_of_many_rows_are_those_of_the_quantizer(fmtc, P, C, e5m2, exponents):  # noqa: F811
    kinds = dict(fmt=fmtc.E5M2 if e5m2 else fmtc.E4M3, scales=fmtc.SCALE_E8M0 if exponents else fmtc.SCALE_F32)
    c = Case(P, C, torch.float32, rows_per_gate=0 if exponents else 60, seed=C + 1)
    q = fmtc.f8_empty(P, C, **kinds)
    h, n, stats = c.forward(fmtc, stats=True)
    h2, _, stats2 = c.forward(fmtc, n_out=q, stats=True)
    want, _ = fmtc.f8_quantize(n, **kinds)
    assert torch.equal(h, h2) and torch.equal(stats, stats2) and torch.equal(q.scales, want.scales)
    assert torch.equal(q.codes.view(torch.uint8), want.codes.view(torch.uint8))


@pytest.mark.parametrize("P, C", [(1, 4096), (6, 100), (33, 1000), (1300, 4096), (9001, 300), (701, 8191), (600, 16384)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("exponents", [False, True])
def test_codes_of_streams_of_16_bits(fmtc, P, C, dtype, exponents):  # noqa: F811
    """n is quantized before it is rounded to the stream's type, so its codes are those that the same values give as an f32
    stream, but for what another order of f32 roundings moves across the middle between two codes: numbers are off by
    1e-6 of their size, codes lie 2^-4 and more of it apart, which is 2e-5 of them; 2e-4 may differ.  (n rounded to bf16 first
    would move some 3 %, to f16 some 0.4 %.)  Values: half a step of a code, 2^-4 of their size or 2^-10 of the scale, and f32
    roundings of h' before it, whose parts are up to 8 times the row's largest: 24 x 2^-24 x 8."""
    kinds = dict(scales=fmtc.SCALE_E8M0 if exponents else fmtc.SCALE_F32)
    c = Case(P, C, dtype, rows_per_gate=5, skip=0.9, scale=0.5, seed=C + 2)
    q = fmtc.f8_empty(P, C, **kinds)
    h, _, _ = c.forward(fmtc, n_out=q)
    h2, _, _ = c.forward(fmtc)
    assert torch.equal(h, h2)
    _, _, n, _, _ = c.want()
    off = (ref.values(q.codes, q.scales, C) - n).abs()
    step = q.scales.cpu().double().t().repeat_interleave(128, 1)[:, :C]
    lost = 24 * 2.0 ** -24 * 8 * n.abs().amax(1, keepdim=True)
    assert (off <= 1.001 * (2.0 ** -4 * n.abs() + 2.0 ** -10 * step) + lost).all()
    c.y, c.h = c.y.float(), c.h.float()
    wide = fmtc.f8_empty(P, C, **kinds)
    c.forward(fmtc, n_out=wide)
    other = int((q.codes.view(torch.uint8) != wide.codes.view(torch.uint8)).sum())
    assert other <= 2e-4 * P * C + 1
    assert torch.allclose(q.scales.float(), wide.scales.float(), rtol=1e-5) or exponents
    assert not q.codes.view(torch.uint8)[:, C:].any()


# rows, channels and rows of a gate: strips of 2 to 9 rows
STRIPS = [(70000, 40, 1), (70000, 100, 3), (20487, 300, 2), (20487, 512, 5), (9001, 1000, 3), (5000, 2000, 4), (2000, 4096, 1), (2000, 4096, 2),
          (2001, 4096, 3), (1501, 4095, 2), (1500, 8192, 3), (1000, 8191, 2), (900, 9001, 1), (900, 9001, 2), (700, 16384, 3)]


@pytest.mark.parametrize("P, C, rows_per_gate", STRIPS)
def test_gradients_of_strips_of_whole_gate_rows(fmtc, P, C, rows_per_gate):  # noqa: F811
    _check_backward(fmtc, Case(P, C, rows_per_gate=rows_per_gate, skip=0.9, scale=0.5, seed=P))


@pytest.mark.parametrize("P, C, rows_per_gate", STRIPS)
@pytest.mark.parametrize("gate", [False, True])
def test_gradients_of_strips_of_a_gate_row_or_none(fmtc, P, C, rows_per_gate, gate):  # noqa: F811
    _check_backward(fmtc, Case(P, C, rows_per_gate=P // 3 + 1 if gate else 0, scale=0.5, gate=gate, seed=P))


@pytest.mark.parametrize("P, C", [(20487, 300), (2001, 4096), (900, 9001)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_gradients_of_strips_in_other_types_and_without_some_parts(fmtc, P, C, dtype):  # noqa: F811
    _check_backward(fmtc, Case(P, C, dtype, dtype, rows_per_gate=2, seed=C))
    _check_backward(fmtc, Case(P, C, dtype, rows_per_gate=2, post=False, seed=C))
    _check_backward(fmtc, Case(P, C, dtype, y=False, seed=C))
    _check_backward(fmtc, Case(P, C, dtype, rows_per_gate=3, seed=C), dh=False)
    _check_backward(fmtc, Case(P, C, dtype, rows_per_gate=3, seed=C), dn=False)


@pytest.mark.parametrize("P, C", [(17 * 4096 + 3, 300), (300000, 16)])
def test_gradients_of_long_strips(fmtc, P, C):  # noqa: F811
    _check_backward(fmtc, Case(P, C, gate=False, scale=0.5, seed=C))
