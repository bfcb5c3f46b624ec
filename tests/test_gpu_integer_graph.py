"""Group norm, products in 8-bit integers, gradients and clipping as they are used together: in one HIP graph replayed between
eager work, on another stream, with workspaces of the caller's, and where a call may not be made."""
import os
import re

import pytest

torch = pytest.importorskip("torch")
import more_reference as ref  # noqa: E402
from paper_1905_10830_amd import binding as fmtc  # noqa: E402

pytestmark = pytest.mark.gpu


def _normal(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s: torch.randn(s, generator=g, device="cuda")


def _size(n):
    return torch.empty(max(256, n), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("maps, pixels, C, G, O", [(1, 1, 64, 8, 40), (2, 196, 96, 8, 200), (1, 9000, 64, 4, 130), (40, 49, 264, 33, 1000)])
def test_all_in_a_graph(maps, pixels, C, G, O):
    normal, P = _normal(8), maps * pixels
    x, dy, head = normal(P, C).bfloat16(), normal(P, C).bfloat16(), normal(P, O)
    weight, bias, w = normal(C), normal(C), fmtc.i8_quantize(normal(O, C))
    kw = dict(rows_per_sample=pixels, act=fmtc.ACT_SILU)
    ws = [_size(fmtc.group_norm_workspace_size(P, C, G, pixels)), _size(fmtc.group_norm_workspace_size(P, C, G, pixels, to_codes=True)),
          _size(fmtc.i8_matmul_workspace_size(P, O, C)), _size(fmtc.i8_linear_workspace_size(P, O, C)),
          _size(fmtc.group_norm_backward_workspace_size(P, C, G, pixels))]

    def step():
        y, stats = fmtc.group_norm(x, G, weight, bias, stats=True, workspace=ws[0], **kw)
        codes, _ = fmtc.group_norm(x, G, weight, bias, out=fmtc.i8_empty(P, C), workspace=ws[1], **kw)
        served = fmtc.i8_matmul(codes, w, workspace=ws[2])
        layer = fmtc.i8_linear(y, w, workspace=ws[3])
        grads = fmtc.group_norm_backward(dy, x, stats, G, weight, bias, workspace=ws[4], **kw)
        held = [head.clone(), grads[1].clone(), grads[2].clone()]
        norm = fmtc.Tensors(held).clip(1.0)
        return (y, stats, codes.codes, codes.scales, served, layer, *grads, norm, *held)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        for t in (x, dy, head):
            t.copy_(normal(*t.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(held, step(), strict=True):
            assert torch.equal(got, want)


def test_a_map_served_and_trained():
    """A norm to the codes of a product is the product of the norm's values, but for their rounding; its gradient reaches the
    product's operand; all gradients are clipped together."""
    normal = _normal(3)
    maps, pixels, C, G, O = 3, 200, 96, 8, 150
    P = maps * pixels
    x, weight, bias = normal(P, C), 1 + 0.2 * normal(C), 0.2 * normal(C)
    kw = dict(rows_per_sample=pixels, act=fmtc.ACT_SILU)
    w = fmtc.i8_quantize(normal(O, C))
    codes, stats = fmtc.group_norm(x, G, weight, bias, out=fmtc.i8_empty(P, C), stats=True, **kw)
    y, same = fmtc.group_norm(x, G, weight, bias, stats=True, **kw)
    assert torch.equal(codes.codes, fmtc.i8_quantize(y).codes)  # (f32 values: nothing is rounded between)
    assert torch.equal(fmtc.i8_matmul(codes, w, dtype=torch.float32), fmtc.i8_linear(y, w))
    assert float((stats - same).abs().max()) <= 2 * ref.U * float(stats.abs().max())  # (in one pass or in two: sums in another order)


@pytest.mark.parametrize("pixels", [196, 40000])
def test_another_stream_and_two_calls_at_once(pixels):
    normal = _normal(5)
    C, G = 64, 8
    xs = [normal(pixels, C).bfloat16() for _ in range(2)]
    w = fmtc.i8_quantize(normal(300, C))
    tensors = [[normal(100000), normal(33)] for _ in range(2)]
    kw = dict(act=fmtc.ACT_RELU, stats=True)

    def work(i):
        y, stats = fmtc.group_norm(xs[i], G, **kw)
        outs = [torch.empty_like(t) for t in tensors[i]]
        return y, stats, fmtc.i8_linear(y, w), fmtc.Tensors(tensors[i], out=outs).clip(1.0), *outs
    want = [work(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append(work(i))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, v in zip(got, want) for a, b in zip(g, v))


def test_calls_that_are_refused():
    normal = _normal(1)
    x, v = normal(12, 16), normal(16)
    w = fmtc.i8_quantize(normal(8, 16))
    bad = [lambda: fmtc.group_norm(x, 5), lambda: fmtc.group_norm(x, 0), lambda: fmtc.group_norm(x, 4, rows_per_sample=5), lambda: fmtc.group_norm(x, 4, act=3),
           lambda: fmtc.group_norm(x, 4, eps=-1.0), lambda: fmtc.group_norm(x, 4, v[:8]), lambda: fmtc.group_norm(x, 4, v, v.bfloat16()),
           lambda: fmtc.group_norm(x, 4, v.bfloat16()), lambda: fmtc.group_norm(x.t(), 4), lambda: fmtc.group_norm(x.cpu(), 4),
           lambda: fmtc.group_norm(x, 4, out=x.bfloat16()), lambda: fmtc.group_norm(x, 4, out=x[:6]), lambda: fmtc.group_norm(x, 4, out=fmtc.i8_empty(12, 15)),
           lambda: fmtc.group_norm(x, 4, out=False), lambda: fmtc.group_norm(x, 4, stats=normal(2, 1, 3)), lambda: fmtc.group_norm(x.double(), 4),
           lambda: fmtc.group_norm_backward(x, x, None, 4), lambda: fmtc.group_norm_backward(x[:6], x, normal(2, 1, 4), 4),
           lambda: fmtc.group_norm_backward(x.bfloat16(), x, normal(2, 1, 4), 4), lambda: fmtc.group_norm_backward(x, x, normal(2, 1, 4), 4, dx=False),
           lambda: fmtc.group_norm_backward(x, x, normal(2, 1, 4), 4, v, workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
           lambda: fmtc.i8_linear(x[:, :15], w), lambda: fmtc.i8_linear(x, w, bias=v[:7]), lambda: fmtc.i8_linear(x, w, bias=v[:8].bfloat16()),
           lambda: fmtc.i8_linear(x, w, out=normal(12, 9)), lambda: fmtc.i8_linear(x, w, dtype=torch.float64), lambda: fmtc.i8_linear(x.cpu(), w),
           lambda: fmtc.i8_matmul(fmtc.i8_quantize(x[:, :15]), w), lambda: fmtc.i8_matmul(w, w, out=normal(8, 8), dtype=torch.bfloat16),
           lambda: fmtc.i8_quantize(x, out=fmtc.i8_empty(11, 16)), lambda: fmtc.i8_quantize(x, out=fmtc.i8_empty(12, 17)), lambda: fmtc.i8_quantize(v),
           lambda: fmtc.i8_empty(3, 0), lambda: fmtc.i8_empty(3, fmtc.I8_DEPTH + 1),
           lambda: fmtc.I8(w.codes[:, :100], w.scales, 16), lambda: fmtc.I8(w.codes, w.scales[:7], 16), lambda: fmtc.I8(w.codes.view(torch.uint8), w.scales, 16),
           lambda: fmtc.I8(w.codes, w.scales, 200), lambda: fmtc.I8(w.codes, w.scales, 0), lambda: fmtc.I8(w.codes.cpu(), w.scales, 16),
           lambda: fmtc.I8(w.codes, w.scales.half(), 16), lambda: fmtc.I8(w.codes.t(), torch.empty(128, device="cuda"), 8)]
    for k, call in enumerate(bad):
        with pytest.raises((ValueError, fmtc.FmtcError)):
            call()
            pytest.fail(f"call {k} was taken")
    torch.cuda.synchronize()


def test_inputs_of_another_stream_are_in_order():
    """The current stream's work is what a call waits for, as of any torch operation."""
    side = torch.cuda.Stream()
    x = torch.zeros((4096, 256), device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            x.add_(1.0)
        x[:, ::2] = -1.0
        y, _ = fmtc.group_norm(x, 1)
    side.synchronize()
    want = ref.group_norm(x, 1, 1, None, None, "none", 1e-5, torch.float32)
    assert bool(((y.double() - want[0]).abs() <= want[1]).all())


def test_the_program_of_the_readme():
    text = open(os.path.join(os.path.dirname(os.path.dirname(__file__)), "README.md")).read()
    code = [c for c in re.findall(r"```python\n(.*?)```", text, re.S) if "i8_linear" in c]
    assert len(code) == 1
    names = {"torch": torch, "fmtc": fmtc}
    exec(code[0], names)
    # two operands off by 0.8 % each (1 / sqrt(12) of 1 / 127 of a row's largest, 3 to 4 times its size)
    want = names["x"].double() @ names["w"].double().t()
    assert float((names["rows"].double() - want).norm() / want.norm()) < 0.02
    want = names["y"].double() @ names["w"].double().t()
    assert float((names["out"].double() - want).norm() / want.norm()) < 0.02
    squares = sum(float(names[k].double().square().sum()) for k in ("dweight", "dshift"))
    assert abs(squares ** 0.5 - min(1.0, float(names["total"]))) < 1e-5
    assert names["dx"].shape == names["x"].shape
