"""Argument checks of the block operators: found on the host, before anything is launched (no GPU needed), and the plain
references of their tests against differences."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")
import f8_reference as ref  # noqa: E402
from paper_1905_10830_amd import binding as fmtc  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fmtc.LIB_PATH):
        from paper_1905_10830_amd import build

        build.build()
    return fmtc.load_library()


SOME = 1 << 20  # an address that is never read


def _f8(**more):
    f = dict(d_codes=SOME, d_scales=SOME, rows=64, depth=256, ld=256, ld_scales=64, format=0, scale=0, block_rows=1)
    return fmtc._F8(**(f | more))


def _refused(lib, status, word, want=None):
    assert status == (fmtc.EINVAL if want is None else want)
    assert word in lib.fmtc_last_error().decode(), lib.fmtc_last_error()


BAD_F8 = [(dict(rows=-1), "is -1 x"), (dict(depth=0), "x 0"), (dict(format=2), "format"), (dict(scale=7), "kind of scale"),
          (dict(block_rows=64), "blocks of 64 rows"), (dict(d_codes=None), "NULL"), (dict(d_scales=None), "NULL"),
          (dict(d_codes=SOME + 8), "alignment"), (dict(d_scales=SOME + 2), "alignment"), (dict(ld=255), "row stride"),
          (dict(ld=264), "row stride"), (dict(depth=257), "row stride"), (dict(ld_scales=63), "stride"), (dict(rows=1 << 31), "x 256")]


@pytest.mark.parametrize("bad, word", BAD_F8)
def test_operands(lib, bad, word):
    good, wrong = _f8(), _f8(**bad)
    for a, b in ((wrong, good), (good, wrong)):
        _refused(lib, lib.fmtc_f8_matmul(a, b, None, SOME, fmtc.F32, 64, 0, None, 0, None), word)


def test_product(lib):
    a, b = _f8(), _f8(block_rows=128, ld_scales=1)
    call = lambda a=a, b=b, bias=None, out=SOME, kind=fmtc.F32, ld=64, add=0, ws=None, size=0: lib.fmtc_f8_matmul(a, b, bias, out, kind, ld, add, ws, size, None)  # noqa: E731
    _refused(lib, call(a=None), "a is NULL")
    _refused(lib, call(b=None), "b is NULL")
    _refused(lib, call(b=_f8(depth=200)), "depths")
    _refused(lib, call(a=b), "blocks of 128")
    _refused(lib, call(b=_f8(scale=1)), "kinds of scale")
    _refused(lib, call(b=_f8(format=1)), "E4M3")
    _refused(lib, call(kind=3), "type 3")
    _refused(lib, call(kind=fmtc.BF16, add=1), "accumulate")
    _refused(lib, call(bias=SOME + 1), "bias")
    _refused(lib, call(out=None), "out is NULL")
    _refused(lib, call(out=SOME + 2), "not aligned")
    _refused(lib, call(ld=63), "row stride")
    assert call(a=_f8(rows=0), out=None) == fmtc.OK and call(b=_f8(rows=0), out=None) == fmtc.OK
    assert lib.fmtc_f8_matmul_workspace_size(0, 4, 4) == 0 and lib.fmtc_f8_matmul_workspace_size(4, 4, 1 << 31) == 0
    size = lib.fmtc_f8_matmul_workspace_size(64, 64, 256)
    if size:
        _refused(lib, call(ws=SOME, size=size - 1), "workspace", fmtc.EBUFSIZE)
        _refused(lib, call(ws=SOME + 1, size=size), "workspace")


def test_quantizer(lib):
    rows, cols = _f8(), _f8(rows=256, depth=64, ld=128, ld_scales=256)
    call = lambda x=SOME, kind=fmtc.BF16, r=64, c=256, ld=256, by_rows=rows, by_cols=cols: lib.fmtc_f8_quantize(x, kind, r, c, ld, by_rows, by_cols, None)  # noqa: E731
    _refused(lib, call(kind=9), "type 9")
    _refused(lib, call(r=-1), "-1 x")
    _refused(lib, call(c=0), "x 0")
    _refused(lib, call(by_rows=None, by_cols=None), "no output")
    _refused(lib, call(x=None), "NULL")
    _refused(lib, call(x=SOME + 1), "not aligned")
    _refused(lib, call(ld=255), "row stride")
    _refused(lib, call(by_rows=_f8(rows=63, ld_scales=64)), "by_rows has another shape")
    _refused(lib, call(by_cols=_f8()), "by_cols has another shape")
    _refused(lib, call(by_rows=_f8(format=1)), "differ")
    assert call(r=0, x=None) == fmtc.OK


def test_gradients(lib):
    w_t = _f8(rows=100, depth=256, block_rows=128, ld_scales=1)
    x_t = _f8(rows=100, depth=64, ld=128, ld_scales=100)
    size = lib.fmtc_f8_matmul_backward_workspace_size(64, 100, 256)
    assert size > 64 * 256 * 2
    call = lambda dy=SOME, kind=fmtc.BF16, P=64, O=256, ld=256, w=w_t, x=x_t, fmt=0, scale=0, dx=SOME, dxk=fmtc.BF16, ldx=100, dw=SOME, ldw=100, db=None, ws=SOME, n=size: lib.fmtc_f8_matmul_backward(dy, kind, P, O, ld, w, x, fmt, scale, dx, dxk, ldx, dw, ldw, db, 0, ws, n, None)  # noqa: E731
    _refused(lib, call(dx=None, dw=None), "no output")
    _refused(lib, call(kind=5), "types")
    _refused(lib, call(fmt=3), "format 3")
    _refused(lib, call(scale=2), "kind of scale 2")
    _refused(lib, call(dy=None), "dy is NULL")
    _refused(lib, call(ld=200), "row stride")
    _refused(lib, call(w=None), "w_t is NULL")
    _refused(lib, call(x=None), "x_t is NULL")
    _refused(lib, call(w=_f8(rows=100, ld_scales=100)), "w_t has to be")
    _refused(lib, call(x=w_t), "x_t has to be")
    _refused(lib, call(scale=1), "w_t has to be")
    _refused(lib, call(w=_f8(rows=99, block_rows=128, ld_scales=1), ldx=99), "w_t has 99 rows, x_t 100")
    _refused(lib, call(ldx=99), "row stride")
    _refused(lib, call(dw=SOME + 2), "not aligned")
    _refused(lib, call(db=SOME + 2), "dbias")
    _refused(lib, call(ws=None), "workspace")
    _refused(lib, call(n=size - 1), "workspace", fmtc.EBUFSIZE)


def test_block_norm(lib):
    base = dict(rows=8, C=64, type=fmtc.BF16, weight_type=fmtc.F32, d_y=SOME, d_h=SOME, ld_y=64, ld_h=64, d_w_post=SOME, d_w_pre=SOME,
                d_gate=SOME, rows_per_gate=4, skip=1.0, scale=1.0, eps=1e-6)
    args = lambda **m: fmtc._Norm(**(base | m))  # noqa: E731
    q = _f8(rows=8, depth=64, ld=128, ld_scales=8)
    call = lambda a=None, h=SOME, ldh=64, n=SOME, ldn=64, codes=None, stats=None, **m: lib.fmtc_block_norm(args(**m) if a is None else None, h, ldh, n, ldn, codes, stats, None)  # noqa: E731
    _refused(lib, call(a=0), "args is NULL")
    for bad, word in ((dict(rows=-1), "-1 rows"), (dict(C=0), "0 channels"), (dict(C=16385), "16385 channels"), (dict(type=4), "type 4"),
                      (dict(weight_type=fmtc.F16), "weights of type"), (dict(d_y=None), "need y"), (dict(rows_per_gate=0), "rows_per_gate"),
                      (dict(d_w_pre=SOME + 2), "not aligned"), (dict(d_h=None), "h is NULL"), (dict(ld_y=63), "row stride"),
                      (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(d_w_pre=None), "n needs w_pre")):
        _refused(lib, call(**bad), word)
    _refused(lib, call(h=None, n=None), "no output")
    _refused(lib, call(ldn=63), "row stride")
    _refused(lib, call(codes=_f8(rows=7, depth=64, ld=128, ld_scales=8)), "n_codes")
    _refused(lib, call(stats=SOME + 1), "stats")
    assert call(rows=0, codes=_f8(rows=0, depth=64, ld=128)) == fmtc.OK
    size = lib.fmtc_block_norm_workspace_size(8, 64, 4)
    assert size and q is not None
    back = lambda stats=SOME, dn=SOME, dh=SOME, dy=SOME, di=SOME, w1=SOME, w2=SOME, dg=SOME, ws=SOME, n=size, **m: lib.fmtc_block_norm_backward(args(**m), stats, dn, 64, dh, 64, dy, 64, di, 64, w1, w2, dg, ws, n, None)  # noqa: E731
    _refused(lib, back(dy=None, di=None, w1=None, w2=None, dg=None), "no output")
    _refused(lib, back(d_w_pre=None), "dn needs w_pre")
    _refused(lib, back(d_w_pre=None, dn=None), "dw_pre needs w_pre")
    _refused(lib, back(d_w_post=None), "dw_post needs w_post")
    _refused(lib, back(d_gate=None), "dgate needs a gate")
    _refused(lib, back(d_y=None, d_w_post=None, d_gate=None), "dy needs y")
    _refused(lib, back(stats=None), "stats is NULL")
    _refused(lib, back(ld_h=63), "row stride")
    _refused(lib, back(dh=SOME + 1), "not aligned")
    _refused(lib, back(ws=None), "workspace")
    _refused(lib, back(n=size - 1), "workspace", fmtc.EBUFSIZE)


def test_reference_gradients_equal_differences():
    """The plain backward pass that GPU tests compare with, against central differences of the plain forward pass: in 64 bits
    a step of 1e-5 is off by 1e-10 of the third derivative and by 1e-16 / 1e-5 from rounding."""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    P, C, R = 7, 20, 3
    t = dict(y=r(P, C), h=r(P, C), w_post=1 + 0.3 * r(C), w_pre=1 + 0.3 * r(C), gate=r(3, C))
    dn, dh = r(P, C), r(P, C)

    def loss(t):
        _, h, n, _, _ = ref.block_norm(t["y"], t["h"], t["w_post"], t["w_pre"], t["gate"], R, 0.9, 0.5, 1e-6)
        return float((dn * n).sum() + (dh * h).sum())

    _, h, _, r_y, r_h = ref.block_norm(t["y"], t["h"], t["w_post"], t["w_pre"], t["gate"], R, 0.9, 0.5, 1e-6)
    got = ref.block_norm_backward(dn, dh, t["y"], h, r_y, r_h, t["w_post"], t["w_pre"], t["gate"], R, 0.9, 0.5)
    for name, grad in zip(("y", "h", "w_post", "w_pre", "gate"), got):
        d = r(*t[name].shape)
        slope = (loss(t | {name: t[name] + 1e-5 * d}) - loss(t | {name: t[name] - 1e-5 * d})) / 2e-5
        assert abs(slope - float((grad * d).sum())) < 1e-7 * (1 + abs(slope)), name


def test_reference_codes_equal_torch():
    g = torch.Generator().manual_seed(2)
    x = torch.randn((50, 300), generator=g)
    for dtype in (torch.float8_e4m3fn, torch.float8_e5m2):
        codes, scales = ref.quantize(x, dtype, exponents=True)
        v = torch.zeros((50, 384))
        v[:, :300] = x
        v = (v.view(50, 3, 128) / scales.t().float()[:, :, None]).view(50, 384)
        assert torch.equal(codes.float(), v.to(dtype).float())
        assert ctypes.sizeof(fmtc._F8) == 64
