"""Training step of early layers with an attention block on their output map's pixels, the block's activations kept in 8 bits.

  python -m paper_2409_09083_amd.token_step [--images 8] [--size 304] [--dtype bf16] [--steps 5]

The early layers run through `harness.Session`; their output map is normalised and turned into token rows, goes through attention and a
two-layer perceptron (both residual), and the loss' gradient comes back the same way into the map's delta and the filters.  What the
block's backward pass needs of its linear layers' inputs, of its second norm's input and of the perceptron's hidden layer is held as
8-bit checkpoints, and the tensors themselves are let go; attention keeps q, k, v and its output, and computes its probabilities again.
Plain matrix products are torch's.
"""
import argparse

import torch

from ftp_synth.configs import conv, pool

from .harness import Session
from .tokens import Attention, Checkpoint, Norm


class TokenBlock:
    """x -> x2 = x + attention(norm(x)) Wo^T, x2 + gelu(norm(x2) W1^T) W2^T for the pixels of a map [batch][channels][pixels]."""

    def __init__(self, batch, pixels, channels, heads, kv_heads, hidden, dtype="f32", block=64, device="cuda", seed=0):
        if channels % heads:
            raise ValueError("%d channels are no multiple of %d heads" % (channels, heads))
        self.rows, self.c, self.hd = batch * pixels, channels, channels // heads
        self.shape, self.heads, self.kv_heads = (batch, pixels, channels), heads, kv_heads
        width = (heads + 2 * kv_heads) * self.hd
        self.norm1 = Norm(batch, pixels, channels, dtype, x_layout="map", device=device)
        self.norm2 = Norm(batch, pixels, channels, dtype, device=device)
        self.attention = Attention(batch, heads, kv_heads, pixels, pixels, self.hd, dtype, device=device)
        kept = lambda cols, outputs=0: Checkpoint(self.rows, cols, dtype, block, outputs, device)        # noqa: E731
        self.kept_n1, self.kept_x2 = kept(channels, width), kept(channels)
        self.kept_n2, self.kept_h, self.kept_a = kept(channels, hidden), kept(hidden), kept(hidden, channels)
        self.out8 = kept(channels, channels)                        # (only in the backward pass, for the weight gradient: attention keeps its output itself)
        g = torch.Generator(device=device).manual_seed(seed)
        t = self.norm1.tdtype

        def weight(n, k):
            return (torch.randn((n, k), generator=g, device=device) * k ** -0.5).to(t)
        self.params = {"wqkv": weight(width, channels), "wo": weight(channels, channels), "w1": weight(hidden, channels),
                       "w2": weight(channels, hidden)}
        for n in ("1", "2"):
            self.params["g" + n], self.params["b" + n] = torch.ones(channels, device=device, dtype=t), torch.zeros(channels, device=device, dtype=t)
        self.grads = {}

    def forward(self, y):
        """y: the early layers' output map [batch][channels][...]; returns the block's output as rows [batch * pixels][channels]."""
        b, n, c = self.shape
        p = self.params
        self.x = y.view(b, c, n).transpose(1, 2)                    # the map seen as tokens
        new = lambda cols: torch.empty((self.rows, cols), dtype=y.dtype, device=y.device)      # noqa: E731
        n1 = new(c)                                                 # (gone when this pass ends, as n2 and a)
        self.norm1.forward(self.x, p["g1"], p["b1"], out=n1.view(self.shape))
        self.kept_n1.pack(n1)
        qkv = (n1 @ p["wqkv"].t()).view(b, n, -1, self.hd)
        self.qkv = qkv.split((self.heads, self.kv_heads, self.kv_heads), 2)
        out = self.attention.forward(*self.qkv).view(-1, c)
        x2 = torch.addmm(self.x.reshape(-1, c), out, p["wo"].t())
        self.kept_x2.pack(x2)
        n2 = new(c)
        self.norm2.forward(x2.view(self.shape), p["g2"], p["b2"], out=n2.view(self.shape))
        self.kept_n2.pack(n2)
        self.kept_h.pack(n2 @ p["w1"].t())
        a = self.kept_h.unpack(act="gelu", out=new(self.kept_h.cols))
        self.kept_a.pack(a)
        return torch.addmm(x2, a, p["w2"].t())

    def backward(self, dz):
        """dz: rows; returns the gradient of y as a map [batch][channels][pixels].  Parameter gradients: self.grads (32 bits)."""
        p, g = self.params, self.grads
        g["w2"] = self.kept_a.wgrad(dz)
        dh = dz @ p["w2"]
        self.kept_h.act_backward(dh, act="gelu", out=dh)
        g["w1"] = self.kept_n2.wgrad(dh)
        dx2, g["g2"], g["b2"] = self.norm2.backward((dh @ p["w1"]).view(self.shape), self.kept_x2, p["g2"])
        dx2 = dx2.view(-1, self.c) + dz
        g["wo"] = self.out8.pack(self.attention.out.view(-1, self.c)).wgrad(dx2)
        dout = (dx2 @ p["wo"]).view(self.shape[0], self.shape[1], self.heads, self.hd)
        dqkv = torch.cat(self.attention.backward(dout, *self.qkv), 2).view(self.rows, -1)
        g["wqkv"] = self.kept_n1.wgrad(dqkv)
        _, g["g1"], g["b1"] = self.norm1.backward((dqkv @ p["wqkv"]).view(self.shape), self.x, p["g1"])
        return self.norm1.dx_buffer + dx2.view(self.shape).transpose(1, 2)

    def update(self, lr):
        for name, w in self.params.items():
            w.add_(self.grads[name].to(w.dtype), alpha=-lr)

    def _kept(self):
        return self.kept_n1, self.kept_x2, self.kept_n2, self.kept_h, self.kept_a

    def kept_bytes(self):
        """Bytes of the 8-bit checkpoints, and of the same values in the block's own type."""
        return (sum(k.codes.nbytes + k.exponents.nbytes for k in self._kept()),
                sum(k.codes.numel() for k in self._kept()) * self.params["wo"].element_size())

    def other_bytes(self):
        """Bytes of what else stays between the passes: q, k, v, attention's output and the statistics; the buffers of gradients and scratch, which every step writes again."""
        n1, n2, a = self.norm1, self.norm2, self.attention
        tensors = [a.out, a.lse, n1.mean, n1.rstd, n2.mean, n2.rstd]
        buffers = [a.dq, a.dk, a.dv, a._ws] + [t for n in (n1, n2) for t in (n.dx_buffer, n.dgamma, n.dbeta, n._ws)] + [t for k in self._kept() for t in (k.dw, k._ws)]
        buffers += [self.out8.codes, self.out8.exponents, self.out8.dw, self.out8._ws]
        return (sum(t.nbytes for t in tensors) + self.qkv[0].untyped_storage().nbytes(), sum(t.nbytes for t in buffers if t is not None))


class TokenStep:
    """Early layers (three convolutions, two pools) with a token block on their output, trained towards a target."""

    def __init__(self, images=8, size=304, dtype="bf16", channels=64, heads=4, kv_heads=2, grid=(2, 2), seed=0):
        layers = (conv(3, 16), pool(16), conv(16, 32), pool(32), conv(32, channels), pool(channels))
        self.early = Session(layers, images, 3, size, size, grid, (2, len(layers)), dtype)
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = self.early.tdtype
        self.early.weights = [(torch.randn((ly.cout, ly.cin, 3, 3), generator=g, device="cuda") * (2 / (9 * ly.cin)) ** 0.5).to(t)
                              if ly.kind == 0 else None for ly in layers]
        self.early.x.copy_(torch.rand(self.early.x.shape, generator=g, device="cuda"))
        b, c, h, w = self.early.out_shape
        self.block = TokenBlock(b, h * w, c, heads, kv_heads, 4 * c, dtype, seed=seed + 1)
        self.target = torch.randn((b * h * w, c), generator=g, device="cuda").to(t)

    def step(self, lr=0.05):
        """Half the mean square distance to the target before the step (a tensor on the device)."""
        self.early.forward()
        d = self.block.forward(self.early.y).float() - self.target
        loss = d.square().mean() / 2
        dmap = self.block.backward((d / d.numel()).to(self.target.dtype))
        self.early.dy.copy_(dmap.view(self.early.dy.shape))
        self.early.backward()
        self.early.sgd_step(lr)
        self.block.update(lr)
        return loss


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--images", type=int, default=8)
    p.add_argument("--size", type=int, default=304)
    p.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    p.add_argument("--steps", type=int, default=5)
    p.add_argument("--lr", type=float, default=0.05)
    a = p.parse_args(argv)
    s = TokenStep(a.images, a.size, a.dtype)
    print("%d images of %d x %d, %d tokens an image, %s" % (a.images, a.size, a.size, s.block.shape[1], a.dtype))
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for i in range(a.steps):
        start.record()
        loss = s.step(a.lr)
        end.record()
        end.synchronize()
        print("step %d: loss %.5f, %.2f ms" % (i, float(loss), start.elapsed_time(end)))
    held, plain = s.block.kept_bytes()
    tensors, buffers = s.block.other_bytes()
    print("kept between the passes: %.1f MB in 8 bits for %.1f MB, and %.1f MB of q, k, v, attention's output and statistics" % (held / 1e6, plain / 1e6, tensors / 1e6))
    print("buffers of gradients and scratch: %.1f MB" % (buffers / 1e6))


if __name__ == "__main__":
    main()
