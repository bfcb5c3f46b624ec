"""The product (fmtc_f8_matmul) at sizes that take each of its kernels: tiles of 128 x 128 with two and with four stages,
tiles of 256 columns, rows by the wavefront in pairs of column tiles, depths in parts with their sums joined; ragged in
every direction, with what lies around the output left as it was."""
import pytest

torch = pytest.importorskip("torch")
import f8_reference as ref  # noqa: E402
from test_gpu_f8 import E4, E5, _check_product, _data, _kinds, _limit, _operands, fmtc  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# rows, columns, depth, and the kernel for bf16 or f16 results / for f32 results
SHAPES = [
    (2, 40, 20000),      # one tile of rows, long depth / the same
    (40, 8200, 1000),    # rows in pairs of column tiles / the same
    (20, 513, 4200),     # 128 x 128 tiles, depth in 11 parts / the same
    (20, 2049, 4200),    # four stages, depth in 11 parts / two stages
    (513, 2049, 1000),   # four stages / rows
    (257, 2500, 300),    # 128 x 128 tiles / the same
    (2049, 2049, 1000),  # 128 x 128 tiles, more than a round / 128 x 256 tiles
    (2049, 4000, 1000),  # 256 x 256 tiles / 128 x 128
    (2049, 2049, 4200),  # 256 x 256 tiles, depth in 2 parts / 128 x 256 tiles
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("exponents", [False, True])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_product_of_each_kernel(fmtc, shape, dtype, exponents, block_rows):  # noqa: F811
    M, N, K = shape
    a, b = _operands(fmtc, M, N, K, E4, exponents, block_rows, 110)
    room = torch.full((M + 1, N + 5), 7.0, dtype=dtype, device="cuda")
    _check_product(fmtc, a, b, dtype, out=room[:M, 2:2 + N], bias=torch.randn(N, generator=torch.Generator().manual_seed(6)))
    assert (room[M:] == 7).all() and (room[:, :2] == 7).all() and (room[:, 2 + N:] == 7).all()


@pytest.mark.parametrize("shape", [(20, 2049, 4200), (2049, 2049, 1000), (2049, 2049, 4200)])
def test_sums_added_to_the_output_of_each_kernel(fmtc, shape):  # noqa: F811
    M, N, K = shape
    a, b = _operands(fmtc, M, N, K, E5, False, 1, 120)
    before = torch.randn((M, N), generator=torch.Generator().manual_seed(7))
    _check_product(fmtc, a, b, torch.float32, out=before.cuda(), add=before, accumulate=True)


@pytest.mark.parametrize("exponents", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_a_nan_stays_in_its_row_and_column_of_a_large_product(fmtc, dtype, exponents):  # noqa: F811
    M, N, K = 2049, 4000, 1000
    x, w = _data(M, K, 130, torch.float32), 0.05 * _data(N, K, 131, torch.float32)
    x[2048, 999], w[3999, 0] = float("nan"), float("nan")
    a, _ = fmtc.f8_quantize(x.cuda(), **_kinds(fmtc, E4, exponents))
    b, _ = fmtc.f8_quantize(w.cuda(), **_kinds(fmtc, E4, exponents))
    bad = torch.isnan(fmtc.f8_matmul(a, b, dtype=dtype))
    assert bad[2048].all() and bad[:, 3999].all() and int(bad.sum()) == M + N - 1


@pytest.mark.parametrize("exponents", [False, True])
def test_gradients_of_a_large_ragged_product(fmtc, exponents):  # noqa: F811
    P, K, O = 2100, 2049, 1000
    dy = 1e-3 * _data(P, O, 140, torch.bfloat16)
    kinds = _kinds(fmtc, E4, exponents)
    _, w_t = fmtc.f8_quantize(0.05 * _data(O, K, 141, torch.float32).cuda(), by_rows=False, by_cols=True, block_rows=128, **kinds)
    _, x_t = fmtc.f8_quantize(_data(P, K, 142).cuda(), by_rows=False, by_cols=True, **kinds)
    dx, dw, _ = fmtc.f8_matmul_backward(dy.cuda(), w_t, x_t, **_kinds(fmtc, E5, exponents))
    rows, wv = ref.values(*ref.quantize(dy, E5, exponents), O), ref.values(w_t.codes, w_t.scales, O)
    cols, xv = ref.values(*ref.quantize(dy.t(), E5, exponents), P), ref.values(x_t.codes, x_t.scales, P)
    for got, a, b in ((dx, rows, wv), (dw, cols, xv)):
        y = a @ b.t()
        assert ((got.cpu().to(torch.float64) - y).abs() <= _limit(a, b, got.dtype, y)).all()


def test_large_products_give_the_same_bits_every_time(fmtc):  # noqa: F811
    for shape in [(2049, 4000, 1000), (2049, 2049, 4200), (20, 2049, 4200)]:
        for dtype in (torch.bfloat16, torch.float32):
            a, b = _operands(fmtc, *shape, E4, False, 128, 150)
            first = fmtc.f8_matmul(a, b, dtype=dtype)
            assert all(torch.equal(first, fmtc.f8_matmul(a, b, dtype=dtype)) for _ in range(4))


@pytest.mark.parametrize("shape", [(600, 520, 512), (2049, 2049, 4200)])
@pytest.mark.parametrize("fmt", [E4, E5])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_power_of_two_scales_at_their_ends(fmtc, shape, fmt, dtype):  # noqa: F811
    """Scales of 2^-127, 2^-126, very large ones, and one that is not a number: a row of a, a column of b."""
    M, N, K = shape
    a, b = _operands(fmtc, M, N, K, fmt, True, 1, 160)
    sa, sb = a.scales.view(torch.uint8), b.scales.view(torch.uint8)
    sa[1, 7], sb[2, 9] = 255, 255
    sa[0, 11], sa[0, 12], sb[0, 3], sa[2, 13], sb[2, 20], sb[1, 21] = 0, 1, 200, 20, 0, 1
    y = fmtc.f8_matmul(a, b, dtype=dtype).cpu().to(torch.float64)
    av, bv = ref.values(a.codes, a.scales, K), ref.values(b.codes, b.scales, K)
    want = av @ bv.t()
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(y), bad) and int(bad.sum()) == M + N - 1
    av, bv = av.nan_to_num(), bv.nan_to_num()
    assert ((y - want).abs() <= _limit(av, bv, dtype, want))[~bad].all()
