"""A block's forward and backward calls (fmtc_block_norm, fmtc_f8_*, and their gradients) in one HIP graph, replayed between
eager work, against the same calls made eagerly; and the README's program."""
import os
import re

import pytest

torch = pytest.importorskip("torch")
from test_gpu_f8 import fmtc  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P, C, O", [(1, 256, 100), (300, 520, 1000)])
def test_a_block_in_a_graph(fmtc, P, C, O):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(8)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    y, h, dy = (normal(P, n).bfloat16() for n in (C, C, O))
    w_post, w_pre, gate = normal(C), normal(C), normal(1, C)
    w, w_t = fmtc.f8_quantize(normal(O, C), by_cols=True, block_rows=128)
    ws = [torch.empty(max(256, n), dtype=torch.uint8, device="cuda") for n in
          (fmtc.f8_matmul_workspace_size(P, O, C), fmtc.f8_matmul_backward_workspace_size(P, C, O), fmtc.block_norm_workspace_size(P, C, P))]

    def step():
        h2, n, stats = fmtc.block_norm(y, h, w_post, w_pre, gate=gate, scale=0.5, stats=True)
        n8, n8_t = fmtc.f8_quantize(n, by_cols=True)
        out = fmtc.f8_matmul(n8, w, workspace=ws[0])
        dn, dw, dbias = fmtc.f8_matmul_backward(dy, w_t, n8_t, bias=True, workspace=ws[1])
        return (h2, out, dw, dbias, *fmtc.block_norm_backward(dn, h2, y, h2, stats, w_post, w_pre, gate=gate, scale=0.5, workspace=ws[2]))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        for t in (y, h, dy):
            t.copy_(normal(*t.shape))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(held, step(), strict=True):
            assert torch.equal(got, want)


def test_the_program_of_the_readme(fmtc):  # noqa: F811
    text = open(os.path.join(os.path.dirname(os.path.dirname(__file__)), "README.md")).read()
    code = [c for c in re.findall(r"```python\n(.*?)```", text, re.S) if "f8_matmul" in c]
    assert len(code) == 1
    names = {"torch": torch, "fmtc": fmtc}
    exec(code[0], names)
    want = names["n"].double().cpu() @ names["w"].double().cpu().t()
    got = names["out"].double().cpu()
    # codes have 4 significant bits: an error of up to 2^-4 of a factor, 2^-5.2 or less in the mean; two factors
    assert float((got - want).norm() / want.norm()) < 2 ** -4
    assert names["dn"].shape == names["n"].shape and names["dw"].shape == names["w"].shape
