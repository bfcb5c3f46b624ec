"""A residual network of pointwise blocks in 8-bit floating point, with its stream stored by the codec.

    python -m paper_1905_10830_amd.blocks [--channels 256] [--hidden 1024] [--blocks 3] [--steps 20] [--bits 6]

Every pixel of a map is a row of the stream h.  A block multiplies the normalised row by two weight matrices with a ReLU
between them; its output is normalised, gated and added to the stream:

    y = W2 relu(W1 n + b1),   u = w_post y / rms(y),   h' = h + gate u,   n' = w_pre' h' / rms(h')

The products take 8-bit codes with a scale per block of 128 (f8_quantize, f8_matmul, f8_matmul_backward), what lies
between them is one call (block_norm, block_norm_backward).  The command trains such a network for a few steps on a
synthetic map, then runs it forward only, one row at a time and as a whole, and stores the last stream with the
feature-map codec (fit_basis, encode, decode).
"""
import argparse
import time

import torch

from . import binding as fmtc

EPS = 1e-6


class Blocks:
    """Parameters (f32) of the blocks and the passes through them.  `scales`: fmtc.SCALE_F32 or fmtc.SCALE_E8M0."""

    def __init__(self, channels, hidden, blocks, scales=fmtc.SCALE_E8M0, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g, device=device)  # noqa: E731
        self.channels, self.scales = channels, scales
        self.params = {"w_pre.0": torch.ones(channels, device=device)}
        for i in range(blocks):
            self.params |= {f"w1.{i}": normal(hidden, channels) / channels ** 0.5, f"b1.{i}": torch.zeros(hidden, device=device),
                            f"w2.{i}": normal(channels, hidden) / hidden ** 0.5,
                            f"w_post.{i}": torch.ones(channels, device=device),
                            f"gate.{i}": torch.full((1, channels), 0.5, device=device),
                            f"w_pre.{i + 1}": torch.ones(channels, device=device)}
        self.blocks = blocks
        self.codes = {}
        self.quantize_weights()

    def quantize_weights(self):
        """Weights as codes, for the products and (transposed) for their gradients: once after every change."""
        for i in range(self.blocks):
            for w in ("w1", "w2"):
                self.codes[f"{w}.{i}"] = fmtc.f8_quantize(self.params[f"{w}.{i}"], by_cols=True, block_rows=fmtc.F8_BLOCK, scales=self.scales)

    def forward(self, h):
        """The stream behind the last block and its normalised rows, without anything kept for gradients: the norm writes
        the codes of the next product itself.  h: bf16 [rows, channels]."""
        p, rows = self.params, len(h)
        codes = lambda: fmtc.f8_empty(rows, self.channels, scales=self.scales, device=h.device)  # noqa: E731
        _, n, _ = fmtc.block_norm(None, h, None, p["w_pre.0"], eps=EPS, h_out=False, n_out=codes())
        for i in range(self.blocks):
            a = fmtc.f8_matmul(n, self.codes[f"w1.{i}"][0], bias=p[f"b1.{i}"])
            r, _ = fmtc.f8_quantize(a.relu_(), scales=self.scales)
            y = fmtc.f8_matmul(r, self.codes[f"w2.{i}"][0])
            h, n, _ = fmtc.block_norm(y, h, p[f"w_post.{i}"], p[f"w_pre.{i + 1}"], gate=p[f"gate.{i}"], eps=EPS,
                                      n_out=codes() if i + 1 < self.blocks else None)
        return h, n

    def forward_backward(self, h, target):
        """-> loss (half the mean square of n - target), gradients of the parameters by name."""
        p, kept = self.params, []
        _, n, stats = fmtc.block_norm(None, h, None, p["w_pre.0"], eps=EPS, h_out=False, stats=True)
        first = (h, stats)
        for i in range(self.blocks):
            n_q, n_t = fmtc.f8_quantize(n, by_cols=True, scales=self.scales)
            r = fmtc.f8_matmul(n_q, self.codes[f"w1.{i}"][0], bias=p[f"b1.{i}"]).relu_()
            r_q, r_t = fmtc.f8_quantize(r, by_cols=True, scales=self.scales)
            y = fmtc.f8_matmul(r_q, self.codes[f"w2.{i}"][0])
            h, n, stats = fmtc.block_norm(y, h, p[f"w_post.{i}"], p[f"w_pre.{i + 1}"], gate=p[f"gate.{i}"], eps=EPS, stats=True)
            kept.append((n_t, r, r_t, y, h, stats))
        off = n.float() - target
        loss = 0.5 * off.square().mean()
        dn, dh, grads = (off / off.numel()).to(n.dtype), None, {}
        for i in reversed(range(self.blocks)):
            n_t, r, r_t, y, h, stats = kept[i]
            dy, dh, grads[f"w_post.{i}"], grads[f"w_pre.{i + 1}"], grads[f"gate.{i}"] = fmtc.block_norm_backward(
                dn, dh, y, h, stats, p[f"w_post.{i}"], p[f"w_pre.{i + 1}"], gate=p[f"gate.{i}"])
            dr, grads[f"w2.{i}"], _ = fmtc.f8_matmul_backward(dy, self.codes[f"w2.{i}"][1], r_t, scales=self.scales)
            da = torch.where(r > 0, dr, 0)
            dn, grads[f"w1.{i}"], grads[f"b1.{i}"] = fmtc.f8_matmul_backward(da, self.codes[f"w1.{i}"][1], n_t, scales=self.scales, bias=True)
        _, _, _, grads["w_pre.0"], _ = fmtc.block_norm_backward(dn, dh, None, first[0], first[1], None, p["w_pre.0"])
        return loss, grads

    def step(self, h, target, rate):
        """One step of gradient descent on normalised gradients.  -> loss"""
        loss, grads = self.forward_backward(h, target)
        for name, g in grads.items():
            self.params[name] -= rate * self.params[name].norm() * g / g.norm().clamp_min(1e-30)
        self.quantize_weights()
        return loss


def _map(pixels, channels, seed):
    """A synthetic stream and a smooth function of it to learn."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rank = max(1, channels // 8)
    z = torch.randn((pixels, rank), generator=g, device="cuda")
    h = z @ (torch.randn((rank, channels), generator=g, device="cuda") / rank ** 0.5)
    target = torch.sin(z @ (torch.randn((rank, channels), generator=g, device="cuda") / rank ** 0.5))
    return h.to(torch.bfloat16), target


def main(argv=None):
    ap = argparse.ArgumentParser(description="trains and runs a network of 8-bit blocks and stores its stream")
    ap.add_argument("--channels", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--side", type=int, default=56)
    ap.add_argument("--bits", type=int, default=6)
    a = ap.parse_args(argv)
    net = Blocks(a.channels, a.hidden, a.blocks)
    h, target = _map(a.side * a.side, a.channels, 1)
    losses = []
    for k in range(a.steps):
        losses.append(float(net.step(h, target, 0.02)))
        print(f"step {k:3d}  loss {losses[-1]:.5f}", flush=True)
    for rows in (1, len(h)):
        x = h[:rows].contiguous()
        net.forward(x)
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(20):
            net.forward(x)
        torch.cuda.synchronize()
        print(f"forward, {rows} rows: {(time.perf_counter() - began) / 20 * 1e6:.0f} us", flush=True)
    stream = net.forward(h)[0].float().view(1, a.side, a.side, a.channels)
    basis = fmtc.fit_basis(stream)
    stored, nbytes = fmtc.encode(basis, stream, a.bits)
    back, err = fmtc.decode(basis, stored, stream.shape, a.bits)
    assert int(err) == 0
    print(f"stream stored at {8 * int(nbytes) / stream.numel():.2f} bits per value ({a.bits}-bit quantizer), "
          f"relative error {float((back - stream).norm() / stream.norm()):.2e}", flush=True)
    return losses


if __name__ == "__main__":
    main()
