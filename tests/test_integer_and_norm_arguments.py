"""Argument checks of the products in 8-bit integers, the group norm and the clipped gradients: found on the host, before
anything is launched (no GPU needed), and the plain references of their tests against differences."""
import ctypes
import math
import os
import random

import pytest

torch = pytest.importorskip("torch")
import more_reference as ref  # noqa: E402
from paper_1905_10830_amd import binding as fmtc  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fmtc.LIB_PATH):
        from paper_1905_10830_amd import build

        build.build()
    return fmtc.load_library()


SOME = 1 << 20  # an address that is never read


def _refused(lib, status, word, want=None):
    assert status == (fmtc.EINVAL if want is None else want)
    assert word in lib.fmtc_last_error().decode(), lib.fmtc_last_error()


def _i8(**more):
    return fmtc._I8(**(dict(d_codes=SOME, d_scales=SOME, rows=64, depth=256, ld=256) | more))


BAD_I8 = [(dict(rows=-1), "is -1 x"), (dict(depth=0), "x 0"), (dict(depth=131072, ld=131072), "x 131072"), (dict(d_codes=None), "NULL"), (dict(d_scales=None), "NULL"),
          (dict(d_codes=SOME + 8), "alignment"), (dict(d_scales=SOME + 2), "alignment"), (dict(ld=255), "row stride"), (dict(ld=264), "row stride"),
          (dict(depth=257), "row stride"), (dict(rows=1 << 31), "x 256")]


@pytest.mark.parametrize("bad, word", BAD_I8)
def test_operands(lib, bad, word):
    good, wrong = _i8(), _i8(**bad)
    for a, b in ((wrong, good), (good, wrong)):
        _refused(lib, lib.fmtc_i8_matmul(a, b, None, SOME, fmtc.F32, 64, None, 0, None), word)
    _refused(lib, lib.fmtc_i8_linear(SOME, fmtc.BF16, 4, 256, wrong, None, SOME, fmtc.F32, 64, SOME, 1 << 30, None), word)
    _refused(lib, lib.fmtc_i8_quantize(SOME, fmtc.BF16, 64, 256, 256, wrong, None), word)


def test_product(lib):
    call = lambda a=_i8(), b=_i8(), bias=None, out=SOME, kind=fmtc.F32, ld=64, ws=None, size=0: lib.fmtc_i8_matmul(a, b, bias, out, kind, ld, ws, size, None)  # noqa: E731, B008
    _refused(lib, call(a=None), "a is NULL")
    _refused(lib, call(b=None), "b is NULL")
    _refused(lib, call(b=_i8(depth=200)), "depths")
    _refused(lib, call(kind=3), "type 3")
    _refused(lib, call(bias=SOME + 1), "bias")
    _refused(lib, call(out=None), "out is NULL")
    _refused(lib, call(out=SOME + 2), "not aligned")
    _refused(lib, call(ld=63), "row stride")
    assert call(a=_i8(rows=0), out=None) == fmtc.OK and call(b=_i8(rows=0), out=None) == fmtc.OK
    for sizes in ((0, 4, 4), (4, 0, 4), (4, 4, 0), (4, 4, 131072), (1 << 31, 4, 4)):
        assert lib.fmtc_i8_matmul_workspace_size(*sizes) == 0 and lib.fmtc_i8_linear_workspace_size(*sizes) == 0


@pytest.mark.parametrize("kind", [fmtc.F32, fmtc.BF16, fmtc.F16])
def test_workspaces(lib, kind):
    M, N, K = 20, 513, 9000  # few tiles of a long depth: in parts, whose sums lie in the workspace
    a, b = _i8(rows=M, depth=K, ld=9088), _i8(rows=N, depth=K, ld=9088)
    for size, call in ((lib.fmtc_i8_matmul_workspace_size(M, N, K), lambda ws, n: lib.fmtc_i8_matmul(a, b, None, SOME, kind, N, ws, n, None)),
                       (lib.fmtc_i8_linear_workspace_size(M, N, K), lambda ws, n: lib.fmtc_i8_linear(SOME, kind, M, K, b, None, SOME, kind, N, ws, n, None)),
                       (lib.fmtc_group_norm_workspace_size(1, 100000, 64, 8, kind, 0), lambda ws, n: lib.fmtc_group_norm(_norm(samples=1, rows_per_sample=100000, C=64, type=kind), SOME, 64, None, None, ws, n, None)),
                       (lib.fmtc_group_norm_workspace_size(2, 50, 64, 8, kind, 1), lambda ws, n: lib.fmtc_group_norm(_norm(samples=2, rows_per_sample=50, C=64, type=kind), None, 0, _i8(rows=100, depth=64, ld=128), None, ws, n, None)),
                       (lib.fmtc_group_norm_backward_workspace_size(2, 50, 64, 8, kind), lambda ws, n: lib.fmtc_group_norm_backward(_norm(samples=2, rows_per_sample=50, C=64, type=kind), SOME, SOME, 64, SOME + 4096, 64, None, None, ws, n, None))):
        assert size > 0
        for ws, n, want in ((SOME, size - 1, fmtc.EBUFSIZE), (SOME, 0, fmtc.EBUFSIZE), (SOME + 1, size, fmtc.EINVAL), (SOME + 128, size, fmtc.EINVAL), (None, size, fmtc.EINVAL)):
            _refused(lib, call(ws, n), "workspace", want)


def test_quantizer_and_layer(lib):
    q = lambda x=SOME, kind=fmtc.BF16, rows=64, cols=256, ld=256, out=_i8(): lib.fmtc_i8_quantize(x, kind, rows, cols, ld, out, None)  # noqa: E731, B008
    _refused(lib, q(out=None), "out is NULL")
    _refused(lib, q(x=None), "x is NULL")
    _refused(lib, q(x=SOME + 1), "not aligned")
    _refused(lib, q(kind=9), "type 9")
    _refused(lib, q(ld=255), "row stride")
    _refused(lib, q(rows=63), "another shape")
    _refused(lib, q(cols=131072), "131072 values")
    assert q(x=None, rows=0, out=_i8(rows=0)) == fmtc.OK
    layer = lambda x=SOME, kind=fmtc.BF16, rows=4, ld=256, w=_i8(), bias=None, out=SOME, out_kind=fmtc.BF16, ld_out=64: lib.fmtc_i8_linear(  # noqa: E731, B008
        x, kind, rows, ld, w, bias, out, out_kind, ld_out, None, 0, None)
    _refused(lib, layer(w=None), "w is NULL")
    _refused(lib, layer(x=None), "x is NULL")
    _refused(lib, layer(kind=4), "type 4")
    _refused(lib, layer(out_kind=4), "type 4")
    _refused(lib, layer(rows=-1), "-1 rows")
    _refused(lib, layer(ld=255), "row stride")
    _refused(lib, layer(ld_out=63), "row stride")
    _refused(lib, layer(bias=SOME + 2), "bias")
    assert layer(rows=0, x=None, out=None) == fmtc.OK and layer(w=_i8(rows=0), out=None) == fmtc.OK


def _norm(**more):
    return fmtc._GroupNorm(**(dict(samples=2, rows_per_sample=10, C=16, groups=8, type=fmtc.BF16, weight_type=fmtc.F32, act=0, eps=1e-5, d_x=SOME, ld_x=64,
                                   d_weight=SOME, d_bias=SOME) | more))


BAD_NORM = [(dict(samples=-1), "-1 samples"), (dict(rows_per_sample=-1), "of -1 rows"), (dict(samples=1 << 20, rows_per_sample=1 << 20), "samples"), (dict(C=0), "0 channels"),
            (dict(C=8200), "8200 channels"), (dict(groups=0), "in 0 groups"), (dict(groups=5), "in 5 groups"), (dict(type=3), "type 3"), (dict(weight_type=fmtc.F16), "weights of type"),
            (dict(act=3), "activation 3"), (dict(act=-1), "activation -1"), (dict(d_x=None), "x is NULL"), (dict(d_x=SOME + 1), "not aligned"), (dict(ld_x=15), "row stride"),
            (dict(d_weight=SOME + 2), "weight or bias"), (dict(d_bias=SOME + 2), "weight or bias")]


@pytest.mark.parametrize("bad, word", BAD_NORM)
def test_norms(lib, bad, word):
    a = _norm(**bad)
    _refused(lib, lib.fmtc_group_norm(a, SOME + 8192, 16, None, None, SOME, 1 << 30, None), word)
    _refused(lib, lib.fmtc_group_norm_backward(a, SOME, SOME, 16, SOME + 8192, 16, None, None, SOME, 1 << 30, None), word)


def test_norm_outputs(lib):
    call = lambda a=_norm(), y=SOME + 8192, ld=16, codes=None, stats=None: lib.fmtc_group_norm(a, y, ld, codes, stats, None, 0, None)  # noqa: E731, B008
    _refused(lib, call(a=None), "args is NULL")
    _refused(lib, call(a=_norm(eps=-1.0)), "eps")
    _refused(lib, call(a=_norm(eps=math.nan)), "eps")
    _refused(lib, call(y=None), "no output")
    _refused(lib, call(y=SOME + 8193), "not aligned")
    _refused(lib, call(ld=15), "row stride")
    _refused(lib, call(y=SOME, ld=16), "another row stride")
    _refused(lib, call(stats=SOME + 2), "stats")
    _refused(lib, call(codes=_i8(rows=19, depth=16)), "codes has to be")
    _refused(lib, call(codes=_i8(rows=20, depth=17)), "codes has to be")
    _refused(lib, call(codes=_i8(rows=20, depth=16, ld=64)), "row stride")
    assert call(a=_norm(samples=0, d_x=None), y=None) == fmtc.OK and call(a=_norm(rows_per_sample=0, d_x=None), y=None) == fmtc.OK
    back = lambda a=_norm(), stats=SOME, dy=SOME, ld_dy=16, dx=SOME + 8192, ld_dx=16, dw=None, db=None: lib.fmtc_group_norm_backward(  # noqa: E731, B008
        a, stats, dy, ld_dy, dx, ld_dx, dw, db, None, 0, None)
    _refused(lib, back(a=None), "args is NULL")
    _refused(lib, back(stats=None), "stats is NULL")
    _refused(lib, back(stats=SOME + 1), "stats")
    _refused(lib, back(dy=None), "dy is NULL")
    _refused(lib, back(ld_dy=15), "row stride")
    _refused(lib, back(ld_dx=15), "row stride")
    _refused(lib, back(dx=None), "no output")
    _refused(lib, back(dx=SOME, ld_dx=16), "another row stride")
    _refused(lib, back(dy=SOME + 512, dx=SOME + 512, ld_dx=32), "another row stride")
    _refused(lib, back(dw=SOME + 2), "dweight")
    _refused(lib, back(db=SOME + 2), "dbias")
    for sizes in ((0, 4, 8, 8), (4, 0, 8, 8), (4, 4, 0, 1), (4, 4, 8, 3), (4, 4, 8, 0), (1 << 20, 1 << 20, 8, 8), (4, 4, 8200, 8)):
        assert lib.fmtc_group_norm_workspace_size(*sizes, fmtc.F32, 1) == 0 and lib.fmtc_group_norm_backward_workspace_size(*sizes, fmtc.F32) == 0
    assert lib.fmtc_group_norm_workspace_size(4, 4, 8, 8, 7, 1) == 0 and lib.fmtc_group_norm_backward_workspace_size(4, 4, 8, 8, 7) == 0


@pytest.mark.parametrize("kind", [fmtc.F32, fmtc.BF16])
@pytest.mark.parametrize("C, groups", [(1, 1), (8, 2), (64, 8), (960, 32), (4104, 3), (8192, 1), (8192, 8192)])
def test_workspaces_of_many_samples(lib, C, groups, kind):
    """What a sample leaves in the workspace is there for as many samples as a launch takes, not for all: up to 2^30 of them."""
    for rows in (1, 2, 50):
        sizes = []
        for samples in (1000, 1 << 14, 1 << 21, (1 << 24) + 5, 1 << 30):
            if samples * rows < 1 << 31:
                sizes.append([lib.fmtc_group_norm_workspace_size(samples, rows, C, groups, kind, to) for to in (0, 1)] +
                             [lib.fmtc_group_norm_backward_workspace_size(samples, rows, C, groups, kind)])
                assert all(n <= 1 << 28 for n in sizes[-1]), (samples, rows, sizes[-1])
        assert sizes[-1] == sizes[-2]


@pytest.mark.parametrize("kind", [fmtc.F32, fmtc.BF16])
@pytest.mark.parametrize("rows, C, groups", [(1, 1, 1), (1, 8, 2), (1, 64, 8), (16, 64, 8), (1, 4096, 1), (2, 960, 32), (1, 8192, 8), (4, 27, 9)])
def test_many_small_samples_take_one_pass(lib, rows, C, groups, kind):
    """They fit the registers of a workgroup: nothing is left in the workspace between two passes (two took 4 to 13 times as long)."""
    for samples in (1 << 13, 10000, 1 << 16, 1 << 20, 1 << 24):
        assert lib.fmtc_group_norm_workspace_size(samples, rows, C, groups, kind, 0) == 0, samples


def test_a_norm_writes_values_or_codes(lib):
    codes = _i8(rows=20, depth=16, ld=128)
    _refused(lib, lib.fmtc_group_norm(_norm(), SOME + 8192, 16, codes, None, SOME, 1 << 20, None), "y and codes")
    _refused(lib, lib.fmtc_group_norm(_norm(), SOME + 8192, 16, codes, SOME + 4096, SOME, 1 << 20, None), "y and codes")


def _list(*entries):
    return (fmtc._Tensor * len(entries))(*(fmtc._Tensor(**(dict(d_in=SOME, d_out=SOME + 8192, n=100, type=fmtc.F32, out_type=fmtc.BF16) | e)) for e in entries))


BAD_LIST = [(dict(n=-1), "-1 values"), (dict(n=1 << 41), "values"), (dict(type=3), "type 3"), (dict(out_type=3), "out_type 3"), (dict(d_in=None), "is NULL"),
            (dict(d_in=SOME + 2), "not aligned"), (dict(d_out=SOME + 8193), "not aligned"), (dict(d_out=SOME), "in place in another type"), (dict(d_out=None), "1 of 2 arrays")]


@pytest.mark.parametrize("bad, word", BAD_LIST)
def test_lists(lib, bad, word):
    for k in range(2):
        entries = _list(bad, {}) if k == 0 else _list({}, bad)
        _refused(lib, lib.fmtc_clip(entries, 2, 1.0, 1.0, 1e-6, SOME, SOME, 1 << 20, None), word)
        assert lib.fmtc_clip_workspace_size(entries, 2) == 0


def test_clip(lib):
    some = _list({}, {})
    call = lambda entries=some, n=2, max_norm=1.0, scale=1.0, eps=1e-6, norm=SOME, ws=None, size=0: lib.fmtc_clip(  # noqa: E731
        entries, n, max_norm, scale, eps, norm, ws, size, None)
    _refused(lib, call(n=-1), "list")
    _refused(lib, call(entries=None), "list")
    _refused(lib, call(norm=SOME + 2), "norm is not aligned")
    for bad in (dict(max_norm=-1.0), dict(max_norm=math.nan), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(eps=-1.0), dict(eps=math.inf)):
        _refused(lib, call(**bad), next(iter(bad)))
    only_norm = _list(dict(d_out=None), dict(d_out=None))
    _refused(lib, call(entries=only_norm, norm=None), "no output")
    assert call(entries=None, n=0, norm=None) == fmtc.OK and call(entries=_list(dict(n=0, d_in=None)), n=1, norm=None) == fmtc.OK
    size = lib.fmtc_clip_workspace_size(some, 2)
    for ws, n, want in ((SOME, size - 1, fmtc.EBUFSIZE), (SOME + 1, size, fmtc.EINVAL), (None, size, fmtc.EINVAL)):
        _refused(lib, call(ws=ws, size=n), "workspace", want)


def test_overlaps():
    """Spans that share memory with a written one of another tensor, against all pairs."""
    rng = random.Random(5)
    for _ in range(3000):
        spans = []
        for k in range(rng.randint(0, 5)):
            start = rng.randint(1, 30)
            spans.append((start, start + rng.randint(1, 9), rng.random() < 0.5, (k, 0)))
        want = any(a[0] < b[1] and b[0] < a[1] and (a[2] or b[2]) for i, a in enumerate(spans) for b in spans[i + 1:])
        assert fmtc._overlap(spans) == want, spans


def test_an_i8_shows_what_the_library_reads():
    q = fmtc.i8_empty(4, 200, device="cpu")
    c = fmtc._i8(q)._obj
    assert (c.d_codes, c.d_scales, c.rows, c.depth, c.ld) == (q.codes.data_ptr(), q.scales.data_ptr(), 4, 200, 256)
    assert fmtc._i8(None) is None
    for name in ("codes", "scales", "rows", "depth"):
        with pytest.raises(AttributeError):
            setattr(q, name, getattr(q, name))
    q.scales.data = torch.empty_like(q.scales)
    with pytest.raises(ValueError, match="scales"):
        fmtc._i8(q)
    q = fmtc.i8_empty(4, 200, device="cpu")
    q.codes.resize_(1 << 22)
    with pytest.raises(ValueError, match="codes"):
        fmtc._i8(q)


def test_structures_are_as_large_as_the_header_says():
    """Four 8-byte fields and two ints behind them, and so on: what a C compiler makes of them."""
    assert [ctypes.sizeof(t) for t in (fmtc._I8, fmtc._GroupNorm, fmtc._Tensor)] == [40, 72, 32]


@pytest.mark.parametrize("act", ref.ACTS)
def test_reference_gradients_are_those_of_the_forward_pass(act):
    g = torch.Generator().manual_seed(0)
    normal = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, dy, w, b = normal(12, 12), normal(12, 12), normal(12), normal(12)
    f = lambda x, w, b: float((ref.group_norm(x, 2, 3, w, b, act, 1e-5, torch.float64)[0] * dy).sum())  # noqa: E731
    grads, _ = ref.group_norm_backward(dy, x, 2, 3, w, b, act, 1e-5)
    step = 1e-6
    for which, (at, grad) in enumerate(zip((x, w, b), grads)):
        for i in range(0, at.numel(), 3):
            up, down = ([t.clone() for t in (x, w, b)] for _ in range(2))
            up[which].view(-1)[i] += step
            down[which].view(-1)[i] -= step
            diff = (f(*up) - f(*down)) / (2 * step)
            assert abs(diff - float(grad.view(-1)[i])) <= 1e-6 * (1 + abs(diff))
