"""The product's workspace: refused where it is too small or not aligned, on the host (no GPU needed)."""
import os

import pytest

pytest.importorskip("torch")
from paper_1905_10830_amd import binding as fmtc  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fmtc.LIB_PATH):
        from paper_1905_10830_amd import build

        build.build()
    return fmtc.load_library()


SOME = 1 << 20  # an address that is never read


@pytest.mark.parametrize("kind", [fmtc.F32, fmtc.BF16, fmtc.F16])
@pytest.mark.parametrize("scale", [fmtc.SCALE_F32, fmtc.SCALE_E8M0])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_refusals(lib, kind, scale, block_rows):
    M, N, K = 20, 513, 4200  # few tiles of a long depth: in parts, whose sums lie in the workspace
    a = fmtc._F8(SOME, SOME, M, K, 4224, M, fmtc.E4M3, scale, 1)
    b = fmtc._F8(SOME, SOME, N, K, 4224, -(-N // block_rows), fmtc.E4M3, scale, block_rows)
    size = lib.fmtc_f8_matmul_workspace_size(M, N, K)
    assert size >= 2 * 4 * M * N
    call = lambda ws, n: lib.fmtc_f8_matmul(a, b, None, SOME, kind, N, 0, ws, n, None)  # noqa: E731
    for ws, n, want in ((SOME, size - 1, fmtc.EBUFSIZE), (SOME, 0, fmtc.EBUFSIZE), (SOME + 1, size, fmtc.EINVAL),
                        (SOME + 128, size, fmtc.EINVAL), (None, size, fmtc.EINVAL)):
        assert call(ws, n) == want
        assert "workspace" in lib.fmtc_last_error().decode()
