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


@pytest.mark.parametrize("exponents", [False, True])
def test_gradients_of_a_product(fmtc, exponents):  # noqa: F811
    """f8_quantize gives no transpose of a matrix without rows; the weights say how many columns dw has."""
    scales = fmtc.SCALE_E8M0 if exponents else fmtc.SCALE_F32
    K, O = 100, 60
    _, w_t = fmtc.f8_quantize(torch.ones((O, K), device="cuda"), by_rows=False, by_cols=True, block_rows=128, scales=scales)
    _, x_t = fmtc.f8_quantize(torch.empty((0, K), device="cuda"), by_cols=True, scales=scales)
    assert x_t is None
    dy = torch.empty((0, O), dtype=torch.bfloat16, device="cuda")
    _leave_nan_behind()
    dx, dw, dbias = fmtc.f8_matmul_backward(dy, w_t, x_t, bias=True, scales=scales)
    assert dx.shape == (0, K)
    assert torch.equal(dw, torch.zeros((O, K), device="cuda")) and torch.equal(dbias, torch.zeros(O, device="cuda"))
    # an output that is given says it too, and is added to where that is wanted
    room = torch.full((O, K + 3), 5.0, device="cuda")
    _, got, none = fmtc.f8_matmul_backward(dy, None, None, dw=room[:, 1:1 + K], accumulate=True, scales=scales)
    assert none is None and (room == 5).all()
    _, got, none = fmtc.f8_matmul_backward(dy, None, None, dw=room[:, 1:1 + K], scales=scales)
    assert none is None and got.shape == (O, K) and not got.any()
    assert (room[:, 0] == 5).all() and (room[:, 1 + K:] == 5).all()
    with pytest.raises(ValueError, match="dw needs x_t"):
        fmtc.f8_matmul_backward(torch.empty((1, O), dtype=torch.bfloat16, device="cuda"), None, None, dw=room[:, 1:1 + K], scales=scales)


def test_a_step_of_a_network_on_no_rows(fmtc):  # noqa: F811
    from paper_1905_10830_amd import blocks

    net = blocks.Blocks(64, 96, 2)
    h = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    _leave_nan_behind()
    _, grads = net.forward_backward(h, torch.empty((0, 64), device="cuda"))
    assert set(grads) == set(net.params)
    for name, g in grads.items():
        assert g.shape == net.params[name].shape and not g.any(), name
