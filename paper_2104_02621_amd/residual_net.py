"""A residual stack of capsule convolutions, trained and served with the library's calls alone: an example.

    python -m paper_2104_02621_amd.residual_net [--steps 30] [--state-bits 8] [--dtype bf16] [--graph]

An entry layer, blocks of norm - convolution - norm, gate, residual sum, and a fully-connected capsule layer.  Between
two convolutions there is one launch each way (`block_norm_fwd`, `block_norm_bwd`): it ends one block and begins the next.
The residual stream is float32; what the layers read and write is of `dtype`.  A training step ends with
`grad_norm` (clipping, and no step where a gradient is not finite) and `AdamW`, which also writes the kernels in
`dtype` that the next step's layers read.  Data are synthetic: seeded images and poses to fit.
"""
from __future__ import annotations

import argparse
import time

from . import capscaps as cc


class ResidualCapsNet:
    """Images [N, size, size, 1, 1, d, d] -> poses [N, 1, 1, classes, 1, d, d]."""

    def __init__(self, channels=16, caps=8, blocks=3, size=16, classes=10, dtype=None, lr=2e-3, weight_decay=0.01,
                 state_bits=8, max_norm=1.0, seed=0):
        import torch
        self.torch, self.dtype, self.blocks = torch, torch.bfloat16 if dtype is None else dtype, blocks
        self.max_norm = max_norm
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def kernel(k, c, m):
            fan_in = k * k * c * caps
            return torch.randn((k, k, c, m, 1, caps, caps), generator=gen, device="cuda").mul_(fan_in ** -0.5)

        width = channels * caps * caps
        self.kernels = ([kernel(3, 1, channels)] + [kernel(3, channels, channels) for _ in range(blocks)]
                        + [kernel(size, channels, classes)])
        self.pre = [torch.ones(width, device="cuda") for _ in range(blocks + 1)]
        self.post = [torch.ones(width, device="cuda") for _ in range(blocks)]
        self.gates = [torch.full((width,), 0.1, device="cuda") for _ in range(blocks)]
        self.params = self.kernels + self.pre + self.post + self.gates
        low = [None if self.dtype == torch.float32 else k.to(self.dtype) for k in self.kernels]
        self.layers = [k if c is None else c for k, c in zip(self.kernels, low)]  # what the convolutions read
        vectors = len(self.params) - len(self.kernels)
        self.opt = cc.AdamW(self.params, lr=lr, state_bits=state_bits, seed=seed, copies=low + [None] * vectors,
                            weight_decay=[weight_decay] * len(self.kernels) + [0.0] * vectors)
        self.control = self.opt.control

    def forward(self, images, save=False):
        """Poses; with `save` also what `backward` needs."""
        low = self.dtype != self.torch.float32
        same = dict(norm_dims=4, dtype=self.dtype, save=save)
        x = cc.conv_fwd(images, self.layers[0], 1, 1)
        first = cc.block_norm_fwd(x, pre_weight=self.pre[0], **same)
        h, kept = first.h, [(x, first)]
        for k in range(self.blocks):
            b = cc.conv_fwd(h, self.layers[k + 1], 1, 1, out16=low)
            # serving overwrites the stream; training keeps it
            r = cc.block_norm_fwd(x, b, pre_weight=self.pre[k + 1], post_weight=self.post[k], gate=self.gates[k],
                                  y=None if save else x, **same)
            kept.append((b, r))
            x, h = r.y, r.h
        poses = cc.conv_fwd(h, self.layers[-1])
        return (poses, kept) if save else poses

    def backward(self, images, kept, dposes):
        """Gradients of all parameters, in the order of `params`."""
        low = self.dtype != self.torch.float32
        dk, dpre, dpost, dgate = [None] * len(self.kernels), [None] * (self.blocks + 1), [], []
        h = kept[-1][1].h
        dk[-1] = cc.conv_bwd_kernel(h, dposes, self.kernels[-1].shape[:2])
        dh, dy = cc.conv_bwd_input(dposes, self.layers[-1], h.shape[1:3], out16=low), None
        for k in range(self.blocks - 1, -1, -1):
            b, r = kept[k + 1]
            g = cc.block_norm_bwd(r.y, b, r.rstd_pre, r.rstd_post, dh, dy, pre_weight=self.pre[k + 1],
                                  post_weight=self.post[k], gate=self.gates[k], norm_dims=4)
            dpre[k + 1] = g.dpre_weight
            dpost.insert(0, g.dpost_weight)
            dgate.insert(0, g.dgate)
            h = kept[k][1].h
            dk[k + 1] = cc.conv_bwd_kernel(h, g.dbranch, (3, 3), 1, 1)
            dh, dy = cc.conv_bwd_input(g.dbranch, self.layers[k + 1], h.shape[1:3], 1, 1, out16=low), g.dx
        x, first = kept[0]
        g = cc.block_norm_bwd(x, None, first.rstd_pre, None, dh, dy, pre_weight=self.pre[0], norm_dims=4)
        dpre[0] = g.dpre_weight
        dk[0] = cc.conv_bwd_kernel(images, g.dx.to(self.dtype), (3, 3), 1, 1)
        return dk + dpre + dpost + dgate

    def loss_and_gradients(self, images, targets):
        """Mean square distance of the poses from `targets`."""
        poses, kept = self.forward(images, save=True)
        off = poses - targets
        return off.square().mean(), self.backward(images, kept, (off * (2.0 / off.numel())).to(self.dtype))

    def step(self, images, targets):
        """One training step; returns the loss before it (on the device)."""
        loss, grads = self.loss_and_gradients(images, targets)
        cc.grad_norm(grads, max_norm=self.max_norm, control=self.control)
        self.opt.step(grads, control=self.control)
        return loss


def synthetic_batch(batch, size, caps, classes, dtype, seed=1):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    images = torch.randn((batch, size, size, 1, 1, caps, caps), generator=gen, device="cuda").to(dtype)
    return images, torch.randn((batch, 1, 1, classes, 1, caps, caps), generator=gen, device="cuda")


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    ap.add_argument("--dtype", choices=("bf16", "fp16", "fp32"), default="bf16")
    ap.add_argument("--graph", action="store_true", help="replay the training step as a HIP graph")
    args = ap.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[args.dtype]
    net = ResidualCapsNet(blocks=args.blocks, dtype=dtype, state_bits=args.state_bits)
    images, targets = synthetic_batch(args.batch, 16, 8, 10, dtype)
    loss = net.step(images, targets)
    print(f"step 1: loss {float(loss):.4f}", flush=True)
    run = lambda: net.step(images, targets)  # noqa: E731
    if args.graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = net.step(images, targets)
        run = lambda: (graph.replay(), captured)[1]  # noqa: E731
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for k in range(2, args.steps + 1):
        loss = run()
        if k % 10 == 0 or k == args.steps:
            print(f"step {k}: loss {float(loss):.4f}", flush=True)
    torch.cuda.synchronize()
    if args.steps > 1:
        print(f"{(time.perf_counter() - begin) * 1e3 / (args.steps - 1):.3f} ms a step, {args.batch} images")
    one = net.forward(images[:1])
    print(f"one image served: poses {tuple(one.shape)}, off by {float((one - targets[:1]).square().mean()):.4f}")


if __name__ == "__main__":
    main()
