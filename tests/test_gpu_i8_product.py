"""Products in 8-bit integers: codes equal to their definition bit for bit, results within the roundings that they have."""
import pytest

torch = pytest.importorskip("torch")
import more_reference as ref  # noqa: E402
from paper_1905_10830_amd import binding as fmtc  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _values(rows, cols, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp(torch.randn((rows, 1), generator=g, device="cuda"))
    return x.to(dtype)


def _operand(rows, depth, seed):
    """codes over their whole range, -128 among them, and scales of very different size"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(-128, 128, (rows, depth), generator=g, device="cuda", dtype=torch.int8)
    return q, torch.exp(2 * torch.randn(rows, generator=g, device="cuda"))


def _close(got, want, bound):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), f"off by {float((off / bound).max()):.2f} of the bound"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows, cols", [(1, 1), (3, 7), (5, 8), (17, 127), (2, 128), (9, 129), (4, 512), (3, 513), (33, 960), (2, 2048),
                                        (2, 2049), (3, 4096), (2, 4100), (1, 8192), (2, 8193), (3, 16384), (2, 16385), (1, 20001), (1, 131071)])
def test_codes(dtype, rows, cols):
    x = _values(rows, cols, dtype)
    q = fmtc.i8_quantize(x)
    codes, scales = ref.codes(x)
    assert torch.equal(q.codes, ref.pad(codes)) and torch.equal(q.scales, scales)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [40, 1000, 4096, 17000])
def test_codes_of_rows_apart_from_each_other(dtype, cols):
    """rows with a stride, beginning at odd places, into codes whose rows are longer than they have to be"""
    wide = _values(5, cols + 13, dtype)
    x = wide[:, 5:5 + cols]
    width = -(-cols // 128) * 128
    store = torch.full((5, width + 64), 77, dtype=torch.int8, device="cuda")
    q = fmtc.I8(store, torch.empty(5, device="cuda"), cols)
    assert fmtc.i8_quantize(x, out=q) is q
    codes, scales = ref.codes(x)
    assert torch.equal(store[:, :width], ref.pad(codes)) and torch.equal(q.scales, scales)
    assert bool((store[:, width:] == 77).all())


def test_codes_at_the_ends_of_the_range():
    big, tiny = torch.finfo(torch.float32).max, 2.0 ** -140
    x = torch.zeros((8, 130), device="cuda")
    x[1, 0], x[1, 129] = big, -big
    x[2, 3] = tiny
    x[3] = torch.arange(130, device="cuda") - 63.5           # halves: to even
    x[3, 0] = 127.0
    x[4, 5], x[4, 6] = float("inf"), 1.0
    x[5, 129] = float("nan")
    x[6, 7] = float("-inf")
    x[7] = 2.0 ** -126
    q = fmtc.i8_quantize(x)
    codes, scales = ref.codes(x)
    assert torch.equal(q.codes, ref.pad(codes))
    assert torch.equal(torch.isnan(q.scales), torch.tensor([r in (4, 5, 6) for r in range(8)], device="cuda"))
    assert torch.equal(q.scales.nan_to_num(0.0), scales.nan_to_num(0.0))
    assert float(q.scales[0]) == 2.0 ** -126 and not bool(q.codes[0].any())
    w = fmtc.i8_quantize(_values(40, 130, torch.float32))
    y = fmtc.i8_matmul(q, w, dtype=torch.float32)
    assert torch.equal(torch.isnan(y).all(1), torch.isnan(q.scales)) and torch.equal(torch.isnan(y).any(1), torch.isnan(q.scales))


@pytest.mark.parametrize("cols", [4, 130, 960, 2048, 4100, 17000])
def test_codes_of_any_nan_are_0(cols):
    """NaN of any sign and payload, quiet and not: a row's codes are 0 and its scale is not a number, the others as they are."""
    x = _values(5, cols, torch.float32)
    want, scales = ref.codes(x)
    payloads = torch.tensor([0x7fc00001, 0x7f800001, 0x7f8000ff, 0x7fffffff, -1, -0x3fffff, -0x7fff81], dtype=torch.int64, device="cuda")
    bits = x.view(torch.int32)
    for row in (1, 3):
        at = torch.arange(row % 2, cols, 2, device="cuda")
        bits[row, at] = payloads[at % len(payloads)].to(torch.int32)
    assert bool(torch.isnan(x[1]).any()) and bool(torch.isnan(x[3]).any())
    q = fmtc.i8_quantize(x)
    assert not bool(q.codes[1].any()) and not bool(q.codes[3].any())
    assert bool(torch.isnan(q.scales[[1, 3]]).all())
    for row in (0, 2, 4):
        assert torch.equal(q.codes[row], ref.pad(want)[row]) and bool(q.scales[row] == scales[row])
    y = fmtc.i8_linear(x, fmtc.i8_quantize(_values(40, cols, torch.float32, 1)))
    assert torch.equal(torch.isnan(y).all(1), torch.isnan(q.scales)) and torch.equal(torch.isnan(y).any(1), torch.isnan(q.scales))


@pytest.mark.parametrize("dtype, bad", [(torch.bfloat16, 0x7f81), (torch.bfloat16, -1), (torch.float16, 0x7c01), (torch.float16, 0x7fff)])
def test_codes_of_any_nan_of_16_bits_are_0(dtype, bad):
    x = _values(3, 300, dtype)
    x.view(torch.int16)[1, ::3] = bad
    assert bool(torch.isnan(x[1]).any())
    q = fmtc.i8_quantize(x)
    assert not bool(q.codes[1].any()) and torch.equal(torch.isnan(q.scales), torch.tensor([False, True, False], device="cuda"))


SIZES = [(1, 1, 1), (1, 17, 130), (2, 33, 129), (7, 100, 1000), (16, 1000, 1111), (17, 1, 8), (17, 24, 1024), (31, 513, 65), (64, 64, 64), (65, 129, 257),
         (100, 4096, 300), (128, 128, 4096), (130, 77, 9000), (255, 257, 127), (257, 255, 1025), (513, 1000, 960), (1000, 2050, 384), (2049, 1027, 130),
         (20, 513, 4200), (300, 300, 12000), (1, 5000, 8192), (1100, 1300, 700), (2500, 2600, 259)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, N, K", SIZES)
def test_products(dtype, M, N, K):
    qa, sa = _operand(M, K, 1)
    qb, sb = _operand(N, K, 2)
    a, b = fmtc.I8(ref.pad(qa), sa, K), fmtc.I8(ref.pad(qb), sb, K)
    bias = torch.randn(N, device="cuda") * 1000 if (M + N) % 2 else None
    got = fmtc.i8_matmul(a, b, bias=bias, dtype=dtype) if dtype != torch.bfloat16 else fmtc.i8_matmul(a, b, bias=bias)
    assert got.dtype == dtype
    want, bound = ref.product(qa, sa, qb, sb, bias, dtype)
    top = torch.finfo(dtype).max
    fits, over = want.abs() + bound < top, want.abs() - bound > top * (1 + torch.finfo(dtype).eps)  # (f16 has results beyond it)
    _close(torch.where(fits, got.double(), 0.0), torch.where(fits, want, 0.0), bound)
    assert torch.equal(torch.where(over, got.double(), 0.0), torch.where(over, torch.sign(want) * float("inf"), 0.0))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("M, N, K", [s for s in SIZES if s[0] * s[1] < 2000000])
def test_products_bit_for_bit(dtype, biased, M, N, K):
    """The sum to f32, times s_a, times s_b, plus the bias, each of them rounded, then to the type of the results."""
    qa, sa = _operand(M, K, 11)
    qb, sb = _operand(N, K, 12)
    sa, sb = sa * 1e-3, sb * 1e-3
    want = (qa.double() @ qb.double().t()).float()  # (whole numbers below 2^53: exact until here)
    want = want * sa[:, None]
    want = want * sb
    bias = torch.randn(N, device="cuda") * float(want.abs().median()) if biased else None
    if biased:
        want = want + bias
    got = fmtc.i8_matmul(fmtc.I8(ref.pad(qa), sa, K), fmtc.I8(ref.pad(qb), sb, K), bias=bias, dtype=dtype)
    assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("M", [1, 40, 700])
def test_longest_depth_does_not_overflow(M):
    """-128 x -128, 131071 times: 2^31 - 2^14"""
    K, N = fmtc.I8_DEPTH, 20
    width = -(-K // 128) * 128
    q = torch.zeros((max(M, N), width), dtype=torch.int8, device="cuda")
    q[:, :K] = -128
    ones = torch.ones(max(M, N), device="cuda")
    y = fmtc.i8_matmul(fmtc.I8(q[:M], ones[:M], K), fmtc.I8(q[:N], ones[:N], K), dtype=torch.float32)
    assert bool((y == float(K * 128 * 128)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, N", [(3, 50), (150, 300), (600, 520)])
def test_results_into_a_part_of_a_larger_tensor(dtype, M, N):
    K = 200
    qa, sa = _operand(M, K, 3)
    qb, sb = _operand(N, K, 4)
    sa, sb = sa * 1e-3, sb * 1e-3
    whole = torch.full((M + 2, N + 9), 7.0, dtype=dtype, device="cuda")
    part = whole[1:M + 1, 3:N + 3]
    wide = torch.nn.functional.pad(qa, (0, 256 + 48 - K))
    wide[:, 256:] = 5  # behind what is read
    assert fmtc.i8_matmul(fmtc.I8(wide, sa, K), fmtc.I8(ref.pad(qb), sb, K), out=part) is part
    want, bound = ref.product(qa, sa, qb, sb, None, dtype)
    _close(part, want, bound)
    part.fill_(7.0)
    assert bool((whole == 7.0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M, N, K", [(1, 4096, 4096), (1, 33, 100), (2, 300, 1025), (3, 64, 20000), (4, 100, 960), (5, 700, 4104), (8, 50, 8192), (13, 130, 511),
                                     (16, 128, 2048), (17, 65, 384), (200, 1000, 960), (1025, 520, 333)])
def test_layer_is_quantizer_and_product(dtype, M, N, K):
    x = _values(M, K + 3, dtype)[:, 1:K + 1]
    qb, sb = _operand(N, K, 5)
    w, bias = fmtc.I8(ref.pad(qb), sb * 1e-4, K), torch.randn(N, device="cuda")
    got = fmtc.i8_linear(x, w, bias=bias)
    assert got.dtype == dtype and torch.equal(got, fmtc.i8_matmul(fmtc.i8_quantize(x), w, bias=bias, dtype=dtype))
    qa, sa = ref.codes(x)
    _close(got, *ref.product(qa, sa, qb, sb * 1e-4, bias, dtype))
    other = fmtc.i8_linear(x, w, dtype=torch.float32)
    assert torch.equal(other, fmtc.i8_matmul(fmtc.i8_quantize(x), w, dtype=torch.float32))


@pytest.mark.parametrize("M", [1, 3, 20])
def test_layer_of_a_row_that_is_not_finite(M):
    x = _values(M, 300, torch.bfloat16)
    x[M - 1, 7] = float("inf")
    w = fmtc.i8_quantize(_values(40, 300, torch.float32))
    y = fmtc.i8_linear(x, w)
    assert bool(torch.isnan(y[M - 1]).all()) and not bool(torch.isnan(y[:M - 1]).any())


def test_more_rows_than_a_launch_takes():
    """A grid has less than 2^32 threads: from 2^22 rows on there are several."""
    for rows in (1 << 22, 2 * (1 << 22) + 3):
        x = _values(rows, 8, torch.bfloat16)
        q = fmtc.i8_quantize(x)
        codes, scales = ref.codes(x)
        assert torch.equal(q.codes[:, :8], codes) and not bool(q.codes[:, 8:].any()) and torch.equal(q.scales, scales)


@pytest.mark.parametrize("M", [1, 3, 12])
def test_more_columns_than_a_launch_takes(M):
    """2^27 and some rows of weights (16 a workgroup of 512 threads)"""
    N, K = (1 << 27) + 37, 6
    store = torch.zeros((N, 128), dtype=torch.int8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for c in range(K):
        store[:, c] = torch.randint(-127, 128, (N,), generator=g, device="cuda", dtype=torch.int8)
    scales = torch.rand(N, generator=g, device="cuda")
    w, bias, x = fmtc.I8(store, scales, K), torch.randn(N, generator=g, device="cuda"), _values(M, K, torch.float32)
    qa, sa = ref.codes(x)
    want = sum(qa[:, c].float()[:, None] * store[:, c].float() for c in range(K))  # (whole numbers below 2^24: exact)
    want = want * sa[:, None]
    want = want * scales
    want = want + bias
    assert torch.equal(fmtc.i8_linear(x, w, bias=bias), want)
    assert torch.equal(fmtc.i8_matmul(fmtc.i8_quantize(x), w, bias=bias, dtype=torch.float32), want)


def test_no_rows():
    w = fmtc.i8_quantize(_values(40, 300, torch.float32))
    x = torch.empty((0, 300), dtype=torch.bfloat16, device="cuda")
    assert fmtc.i8_quantize(x).codes.shape == (0, 384)
    assert fmtc.i8_linear(x, w).shape == (0, 40) and fmtc.i8_matmul(fmtc.i8_quantize(x), w).shape == (0, 40)
    none = fmtc.i8_empty(0, 300)
    assert fmtc.i8_linear(x[:0], none).shape == (0, 0) and fmtc.i8_matmul(w, none).shape == (40, 0)


@pytest.mark.parametrize("M, N, K", [(20, 513, 4200), (1, 512, 4096), (600, 700, 300)])
def test_the_same_numbers_in_every_run(M, N, K):
    x = _values(M, K, torch.float32)
    w = fmtc.i8_quantize(_values(N, K, torch.float32, 1))
    first = fmtc.i8_linear(x, w)
    assert all(torch.equal(fmtc.i8_linear(x, w), first) for _ in range(5))
