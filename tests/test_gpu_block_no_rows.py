"""Gradients of a batch without rows: sums over rows are 0, whatever the memory held before."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_block_norm import Case, fmtc  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def _leave_nan_behind():
    """Blocks of the allocator's smallest size, full of NaN, for the next small tensors."""
    held = [torch.full((128,), float("nan"), device="cuda") for _ in range(32)]
    torch.cuda.synchronize()
    del held


@pytest.mark.parametrize("rows_per_gate, gates", [(0, 1), (1, 1), (4, 3)])
@pytest.mark.parametrize("weights", [torch.float32, torch.bfloat16])
def test_gradient_of_a_gate(fmtc, rows_per_gate, gates, weights):  # noqa: F811
    c = Case(0, 100, weights=weights, rows_per_gate=rows_per_gate)
    c.gate = torch.ones((gates, 100), dtype=weights)
    h, _, stats = c.forward(fmtc, stats=True)
    on = c.on
    inputs = [on(t) for t in (c.dn, c.dh, c.y)], [on(t) for t in (c.w_post, c.w_pre, c.gate)]
    _leave_nan_behind()
    got = fmtc.block_norm_backward(*inputs[0], h, stats, *inputs[1][:2], gate=inputs[1][2], **c.more)
    assert got[0].shape == got[1].shape == (0, 100)
    assert got[4].shape == (gates, 100) and got[4].dtype == torch.float32
    for g in got[2:]:
        assert torch.equal(g, torch.zeros_like(g))
