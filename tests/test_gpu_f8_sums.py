"""What the product's sums lose (fmtc_f8_matmul), for every type of result: over all results with operands of one size, of one
sign and with channels far larger than the others, and value by value where a group of products is made to lose the most."""
import pytest

torch = pytest.importorskip("torch")
import f8_reference as ref  # noqa: E402
from test_gpu_f8 import E4, E5, TYPES, _kinds, _limit, fmtc  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def _operands(kind, M, N, K):
    g = torch.Generator().manual_seed(170)
    x, w = torch.randn((M, K), generator=g), torch.randn((N, K), generator=g)
    if "channels" in kind:
        x *= torch.where(torch.rand(K, generator=g) < 0.02, 100.0, 1.0)
    if "one sign" in kind:
        x, w = x.abs(), w.abs()
    if "relu" in kind:
        x = x.relu()
    return x, w


# the share of a result's norm that 8-bit instructions may lose, as the header has it
LOST = {"any sign": 3e-5, "one sign": 3e-5, "relu": 3e-5, "large channels": 1e-4, "one sign, large channels": 1e-4}


@pytest.mark.parametrize("M", [16, 300])
@pytest.mark.parametrize("kind", LOST)
@pytest.mark.parametrize("exponents", [False, True])
@pytest.mark.parametrize("fmt", [E4, E5])
def test_sums_over_all_results(fmtc, M, kind, exponents, fmt):  # noqa: F811
    """Rounding to the result's type has no relation to what the sums lost: the squares of the two add up.  1 % for the chance
    in the rounding of 300 x 300 numbers or 16 x 2000 (its norm is known to about 1 / sqrt(2 x 32000) = 0.4 %).  f32: as
    many roundings of 2^-24 of the running sum as blocks of 128 (16), in the mean over signs less: 1e-6."""
    N, K = (2000 if M == 16 else 300), 2048
    x, w = _operands(kind, M, N, K)
    a, _ = fmtc.f8_quantize(x.cuda(), **_kinds(fmtc, fmt, exponents))
    b, _ = fmtc.f8_quantize(w.cuda(), block_rows=128, **_kinds(fmtc, E4, exponents))
    y = ref.values(a.codes, a.scales, K) @ ref.values(b.codes, b.scales, K).t()
    for dtype in TYPES:
        off = float((fmtc.f8_matmul(a, b, dtype=dtype).cpu().double() - y).norm() / y.norm())
        rounding = float((y.to(dtype).double() - y).norm() / y.norm())
        lost = 1e-6 if dtype == torch.float32 else LOST[kind]
        assert off <= 1.01 * (rounding ** 2 + lost ** 2) ** 0.5, (dtype, off, rounding)


@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("small", [2.0 ** -13, 2.0 ** -13 * 0.9375, 2.0 ** -12, 2.0 ** -14, 1.0])
@pytest.mark.parametrize("cancel", [False, True])
@pytest.mark.parametrize("exponents", [False, True])
def test_groups_that_lose_the_most(fmtc, M, small, cancel, exponents):  # noqa: F811
    """One product of every 8 is 1, the others are about what an instruction no longer sees beside it; or the large ones cancel
    and what is left over are the small ones.  Value by value within what the sums may lose."""
    N, K = 150, 1024
    x, w = torch.full((M, K), 2.0 ** -6), torch.full((N, K), 2.0 ** 6 * small)
    x[:, ::8], w[:, ::8] = 1.0, 1.0
    if cancel:
        x[:, ::16] = -1.0
    x *= 1.0 + torch.arange(M)[:, None] % 3 / 8
    a, _ = fmtc.f8_quantize(x.cuda(), **_kinds(fmtc, E4, exponents))
    b, _ = fmtc.f8_quantize(w.cuda(), block_rows=128, **_kinds(fmtc, E4, exponents))
    av, bv = ref.values(a.codes, a.scales, K), ref.values(b.codes, b.scales, K)
    y = av @ bv.t()
    for dtype in TYPES:
        off = (fmtc.f8_matmul(a, b, dtype=dtype).cpu().double() - y).abs()
        limit = _limit(av, bv, dtype, y)
        assert (off <= limit).all(), (dtype, float((off / limit).max()))
