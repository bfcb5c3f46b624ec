"""Sizes of the norms' workspace at the ends of what a call may say (no GPU needed)."""
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


@pytest.mark.parametrize("C", [40, 300, 4096, 16384])
@pytest.mark.parametrize("rows", [1, 2, 100, 70000])
@pytest.mark.parametrize("many", [(1 << 63) - 1, (1 << 63) - 2, 1 << 62, (1 << 32) + 1])
def test_a_gate_row_for_more_rows_than_there_are(lib, rows, C, many):
    """is one for all of them, however many it says."""
    one = lib.fmtc_block_norm_workspace_size(rows, C, rows)
    assert one >= 2 * 4 * C
    assert lib.fmtc_block_norm_workspace_size(rows, C, rows + 1) == one
    assert lib.fmtc_block_norm_workspace_size(rows, C, many) == one


@pytest.mark.gpu
@pytest.mark.parametrize("many", [(1 << 63) - 1, 1 << 63, (1 << 64) + 2, 1 << 100])
def test_calls_with_a_gate_row_for_any_number_of_rows(many):
    import torch

    from test_gpu_block_norm import Case

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    for P, C in ((1, 40), (7, 300), (600, 4096)):
        c = Case(P, C, rows_per_gate=0, seed=P)
        on = c.on
        runs = []
        for n in (0, many):
            c.more["rows_per_gate"] = n
            h, out, stats = c.forward(fmtc, stats=True)
            runs.append((h, out, stats, *fmtc.block_norm_backward(on(c.dn), on(c.dh), on(c.y), h, stats, on(c.w_post), on(c.w_pre),
                                                                  gate=on(c.gate), **c.more)))
        assert all(torch.equal(a, b) for a, b in zip(*runs, strict=True))
