"""The network of 8-bit blocks behind a stem (group norm, activation, product), its clipped step and its form in integers,
against the same network in 64 bits by torch's autograd."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
MAPS, PIXELS, INPUTS, GROUPS = 4, 125, 48, 6


@pytest.fixture(scope="module")
def blocks():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_10830_amd import blocks

    return blocks


def _plain(net, x, target):
    p = {k: v.detach().cpu().double().requires_grad_() for k, v in net.params.items()}
    rms = lambda v: torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6)  # noqa: E731
    v = x.cpu().double().view(MAPS, PIXELS, GROUPS, -1)
    v = (v - v.mean((1, 3), keepdim=True)) / torch.sqrt(v.var((1, 3), unbiased=False, keepdim=True) + 1e-5)
    z = v.view(MAPS * PIXELS, INPUTS) * p["stem.weight"] + p["stem.bias"]
    h = (z * torch.sigmoid(z)) @ p["ws"].t() + p["bs"]
    n = p["w_pre.0"] * h / rms(h)
    for i in range(net.blocks):
        y = torch.relu(n @ p[f"w1.{i}"].t() + p[f"b1.{i}"]) @ p[f"w2.{i}"].t()
        h = h + p[f"gate.{i}"] * p[f"w_post.{i}"] * y / rms(y)
        n = p[f"w_pre.{i + 1}"] * h / rms(h)
    loss = 0.5 * (n - target.cpu().double()).square().mean()
    loss.backward()
    return h.detach(), n.detach(), float(loss.detach()), {k: v.grad for k, v in p.items()}


def _rel(a, b):
    return float((a.cpu().double() - b).norm() / b.norm())


def _network(blocks, scales=1):
    net = blocks.Blocks(200, 300, 2, scales=scales, inputs=INPUTS, groups=GROUPS)
    g = torch.Generator(device="cuda").manual_seed(4)
    net.params["stem.weight"] += 0.2 * torch.randn(INPUTS, generator=g, device="cuda")
    net.params["stem.bias"] += 0.2 * torch.randn(INPUTS, generator=g, device="cuda")
    return net, *blocks._map(MAPS * PIXELS, INPUTS, 3, 200)


@pytest.mark.parametrize("scales", [0, 1])
def test_network_follows_the_one_in_64_bits(blocks, scales):
    """As without a stem: operands in 8-bit floating point are off by 2^-5.5 of their size each; the stem's product adds 3 % to
    the stream (two operands, half of it squared together), to its output and to the directions of gradients before it."""
    net, x, target = _network(blocks, scales)
    want_h, want_n, want_loss, want = _plain(net, x, target)
    got_h, got_n = net.forward(x, rows_per_sample=PIXELS)
    assert _rel(got_h, want_h) < 0.06 and _rel(got_n, want_n) < 0.06
    loss, grads = net.forward_backward(x, target, rows_per_sample=PIXELS)
    assert abs(float(loss) - want_loss) < 0.06 * want_loss
    assert set(grads) == set(want)
    for name, g in want.items():
        assert grads[name].shape == g.shape
        cos = float((grads[name].cpu().double() * g).sum() / (grads[name].cpu().double().norm() * g.norm()))
        assert cos > 0.96, (name, cos)


def test_integers_follow_the_network_in_64_bits(blocks):
    """A code is off by 1 / sqrt(12) of a step of 1 / 127 of the row's largest, which is 3 to 4 times the row's size: 0.8 % of
    each operand, ten operands on the way to the last row: 2.6 % if all of it reached the end."""
    net, x, target = _network(blocks)
    want_h, want_n, _, _ = _plain(net, x, target)
    net.quantize_integers()
    got_h, got_n = net.forward_integers(x, rows_per_sample=PIXELS)
    assert _rel(got_h, want_h) < 0.03 and _rel(got_n, want_n) < 0.03
    one, _ = net.forward_integers(x[:PIXELS], rows_per_sample=PIXELS)
    assert torch.equal(one, got_h[:PIXELS])  # sums of integers: a map's rows are the same alone


def test_clipped_step(blocks):
    """The step that is taken is the gradients', all shortened by one factor, to at most the norm that is given."""
    net, x, target = _network(blocks)
    _, grads = net.forward_backward(x, target, rows_per_sample=PIXELS)
    norm = sum(float(g.double().square().sum()) for g in grads.values()) ** 0.5
    for max_norm in (0.1 * norm, 10 * norm):
        net, x, target = _network(blocks)
        before = {k: v.clone() for k, v in net.params.items()}
        net.step(x, target, 0.5, rows_per_sample=PIXELS, max_norm=max_norm)
        factor = 0.5 * min(1.0, max_norm / (norm + 1e-6))
        for name, g in grads.items():
            # the sum's own rounding, of values up to the parameter's
            want = before[name].double() - factor * g.double()
            assert bool(((net.params[name].double() - want).abs() <= 2.0 ** -23 * (want.abs() + factor * g.double().abs())).all()), name


def test_without_a_stem_nothing_changed(blocks):
    """The same weights for the same seed, whether there is a stem behind them or not."""
    plain, stem = blocks.Blocks(64, 96, 2), blocks.Blocks(64, 96, 2, inputs=16, groups=2)
    assert all(torch.equal(v, stem.params[k]) for k, v in plain.params.items())


def test_the_command_runs(blocks, capsys):
    losses = blocks.main(["--channels", "128", "--hidden", "256", "--blocks", "2", "--steps", "5", "--side", "20", "--inputs", "32", "--max-norm", "1"])
    assert len(losses) == 5
    out = capsys.readouterr().out
    assert "bits per value" in out and "forward in integers, 400 rows" in out
