"""Gradients of a product (fmtc_f8_matmul_backward), all values of an output together: their distance from the plain form is that
of rounding and of what sums lose, so that nothing of the depth is left out or counted twice."""
import pytest

torch = pytest.importorskip("torch")
import f8_reference as ref  # noqa: E402
from test_gpu_f8 import E4, E5, HALF_ULP, TYPES, _data, _kinds, fmtc  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P, K, O", [(1, 200, 70), (127, 60, 300), (128, 256, 128), (333, 190, 257), (1000, 384, 512), (2100, 2049, 1000),
                                     (20000, 64, 64), (30000, 100, 16)])
@pytest.mark.parametrize("exponents", [False, True])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("dtype", TYPES)
def test_distance_of_all_values(fmtc, P, K, O, exponents, fmt, dtype):  # noqa: F811
    """Half a unit of the type at most and 3e-5 beside it in bf16 and f16; f32 1e-6 (a rounding of 2^-24 for each block of the
    depth, in the mean over signs far fewer).  One of 1000 products left out is 3e-2."""
    dy = (1e-3 * _data(P, O, 180, torch.float32)).to(dtype)
    kinds = _kinds(fmtc, E4, exponents)
    _, w_t = fmtc.f8_quantize(0.05 * _data(O, K, 181, torch.float32).cuda(), by_rows=False, by_cols=True, block_rows=128, **kinds)
    _, x_t = fmtc.f8_quantize(_data(P, K, 182).cuda(), by_rows=False, by_cols=True, **kinds)
    dx, dw, dbias = fmtc.f8_matmul_backward(dy.cuda(), w_t, x_t, bias=True, **_kinds(fmtc, fmt, exponents))
    rows, wv = ref.values(*ref.quantize(dy, fmt, exponents), O), ref.values(w_t.codes, w_t.scales, O)
    cols, xv = ref.values(*ref.quantize(dy.t(), fmt, exponents), P), ref.values(x_t.codes, x_t.scales, P)
    for got, y in ((dx, rows @ wv.t()), (dw, cols @ xv.t()), (dbias, dy.double().sum(0))):
        off = float((got.cpu().double() - y).norm() / y.norm())
        assert off <= (1e-6 if got.dtype == torch.float32 else HALF_ULP[got.dtype] + 3e-5), (got.dtype, tuple(got.shape), off)
