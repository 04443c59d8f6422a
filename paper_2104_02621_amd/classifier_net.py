"""A classifier of capsule convolutions with group norms and a head over many classes, trained by class or by a teacher's top
logits: an example.

    python -m paper_2104_02621_amd.classifier_net [--steps 30] [--classes 5000] [--distill] [--dtype bf16] [--graph]

Layers of convolution - group norm - activation, a fully-connected capsule layer whose capsules are a row of features, and a
linear head, whose logits are never kept.  A training step ends with `grad_norm` and `AdamW`, as in residual_net.  Data are
synthetic: seeded images and classes; the teacher is a wider net of the same kind.
"""
from __future__ import annotations

import argparse
import time

from . import capscaps as cc


class CapsClassifier:
    """Images [N, size, size, 1, 1, d, d] -> a loss for each, over `classes`."""

    def __init__(self, channels=8, caps=8, layers=2, size=16, features=4, classes=5000, dtype=None, lr=2e-3, max_norm=1.0,
                 seed=0):
        import torch
        self.torch, self.dtype, self.depth, self.groups = torch, torch.bfloat16 if dtype is None else dtype, layers, channels
        self.max_norm, self.width = max_norm, features * caps * caps
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(fan_in, *shape):
            return torch.randn(shape, generator=gen, device="cuda").mul_(fan_in ** -0.5)

        def kernel(k, c, m):
            return normal(k * k * c * caps, k, k, c, m, 1, caps, caps)

        position = channels * caps * caps
        self.kernels = ([kernel(3, 1, channels)] + [kernel(3, channels, channels) for _ in range(layers - 1)]
                        + [kernel(size, channels, features)])
        self.head = normal(self.width, classes, self.width)
        self.weights = [torch.ones(position, device="cuda") for _ in range(layers)]
        self.biases = [torch.zeros(position, device="cuda") for _ in range(layers)]
        self.head_bias = torch.zeros(classes, device="cuda")
        matrices = self.kernels + [self.head]
        self.params = matrices + self.weights + self.biases + [self.head_bias]
        low = [None if self.dtype == torch.float32 else p.to(self.dtype) for p in matrices]
        vectors = len(self.params) - len(matrices)
        # what the layers read
        *self.layers, self.classifier = [p if c is None else c for p, c in zip(matrices, low)]
        self.opt = cc.AdamW(self.params, lr=lr, copies=low + [None] * vectors,
                            weight_decay=[0.01] * len(matrices) + [0.0] * vectors)
        self.control = self.opt.control

    def features(self, images, save=False):
        """Rows of features [N, width]; with `save` also what `backward` needs."""
        low = self.dtype != self.torch.float32
        h, kept = images, []
        for k in range(self.depth):
            x = cc.conv_fwd(h, self.layers[k], 1, 1)  # float32, normalised before it is rounded
            r = cc.group_norm_fwd(x, self.groups, weight=self.weights[k], bias=self.biases[k], act="silu", channel_dims=4,
                                  dtype=self.dtype, save=save)
            kept.append((h, x, r))
            h = r.y
        rows = cc.conv_fwd(h, self.layers[-1], out16=low).view(len(images), self.width)
        return (rows, kept + [h]) if save else rows

    def _backward(self, kept, g):
        """Gradients of all parameters, in the order of `params`, from those of the head."""
        low = self.dtype != self.torch.float32
        dk, dw, db = [None] * len(self.kernels), [None] * self.depth, [None] * self.depth
        h = kept[-1]
        shape = (len(h), 1, 1) + tuple(self.kernels[-1].shape[3:5]) + (h.shape[5], self.kernels[-1].shape[6])
        d = g.dx.view(shape)
        dk[-1] = cc.conv_bwd_kernel(h, d, self.kernels[-1].shape[:2])
        dh = cc.conv_bwd_input(d, self.layers[-1], h.shape[1:3], out16=low)
        for k in range(self.depth - 1, -1, -1):
            before, x, r = kept[k]
            n = cc.group_norm_bwd(x, self.groups, r.mean, r.rstd, dh, weight=self.weights[k], bias=self.biases[k], act="silu",
                                  channel_dims=4)
            dw[k], db[k] = n.dweight, n.dbias
            dk[k] = cc.conv_bwd_kernel(before, n.dx, (3, 3), 1, 1)
            if k:
                dh = cc.conv_bwd_input(n.dx, self.layers[k], before.shape[1:3], 1, 1, out16=low)
        return dk + [g.dweight] + dw + db + [g.dbias]

    def loss_and_gradients(self, images, targets):
        """The mean cross entropy of the images that have a target (one of the classes; -1: none)."""
        rows, kept = self.features(images, save=True)
        r = cc.class_loss_fwd(rows, self.classifier, targets, bias=self.head_bias)
        share = 1.0 / (targets >= 0).sum().clamp(min=1).float()
        g = cc.class_loss_bwd(rows, self.classifier, targets, r.loss, r.lse, share, bias=self.head_bias)
        return r.loss.sum() * share, self._backward(kept, g)

    def distill_loss_and_gradients(self, images, teacher, temperature=2.0):
        """The mean distance from a teacher's top logits (what `top` returns)."""
        rows, kept = self.features(images, save=True)
        same = dict(bias=self.head_bias, temperature=temperature)
        r = cc.distill_loss_fwd(rows, self.classifier, *teacher, **same)
        share = self.torch.full((), 1.0 / len(images), device=rows.device)
        g = cc.distill_loss_bwd(rows, self.classifier, *teacher, r.lse, r.logq, share, **same)
        return r.loss.mean(), self._backward(kept, g)

    def step(self, images, targets=None, teacher=None):
        """One training step; returns the loss before it (on the device)."""
        loss, grads = (self.loss_and_gradients(images, targets) if teacher is None
                       else self.distill_loss_and_gradients(images, teacher))
        cc.grad_norm(grads, max_norm=self.max_norm, control=self.control)
        self.opt.step(grads, control=self.control)
        return loss

    def top(self, images, k):
        """The largest k logits of each image: (classes, logits)."""
        logits = self.features(images).float() @ self.head.T + self.head_bias
        values, index = logits.topk(k, 1)
        return index, values


def synthetic_batch(batch, size, caps, classes, dtype, seed=1):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    images = torch.randn((batch, size, size, 1, 1, caps, caps), generator=gen, device="cuda").to(dtype)
    return images, torch.randint(0, classes, (batch,), generator=gen, device="cuda")


def main(argv=None):
    import torch
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--classes", type=int, default=5000)
    ap.add_argument("--distill", action="store_true", help="learn from a teacher's 32 largest logits")
    ap.add_argument("--dtype", choices=("bf16", "fp16", "fp32"), default="bf16")
    ap.add_argument("--graph", action="store_true", help="replay the training step as a HIP graph")
    args = ap.parse_args(argv)
    dtype = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}[args.dtype]
    net = CapsClassifier(classes=args.classes, dtype=dtype)
    images, targets = synthetic_batch(args.batch, 16, 8, args.classes, dtype)
    teacher = None
    if args.distill:
        teacher = CapsClassifier(channels=16, classes=args.classes, dtype=dtype, seed=7).top(images, min(32, args.classes))
    run = lambda: net.step(images, targets, teacher)  # noqa: E731
    loss = run()
    print(f"step 1: loss {float(loss):.4f}", flush=True)
    if args.graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = net.step(images, targets, teacher)
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
    one = cc.class_loss_fwd(net.features(images[:1]), net.classifier, targets[:1], bias=net.head_bias)
    print(f"one image scored: probability of its class {float(torch.exp(-one.loss)):.2e}")


if __name__ == "__main__":
    main()
