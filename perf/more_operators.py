"""Performance cases of what ends a stack of capsule layers: the group norm with its activation, the softmax cross
entropy of a linear head over many classes, and distillation from a teacher's top logits through such a head.

`run` computes them in plain torch operations in 32 bits, or, with `own`, through the library's entry points.
`listed()` holds fixed cases; `draw(rng)` makes more of the ranges they stand for; `exact` computes the same from
the definitions in 64 bits.

Notation.  Group norm: x [images, positions, width], `groups` groups of width / groups neighbouring columns, each
normalised over its columns and an image's positions;  y = act(xn weight + bias).
Head: rows x [rows, width], weight [classes, width], bias [classes];  z = x weight^T + bias.
    class loss      log(sum(exp(z))) - z[target];  a row whose target is no class is left out
    distillation    tau^2 sum_k t_k (log t_k - log q_k), t the softmax of the teacher's `top` logits / tau, q that of all z / tau;
                    entries whose index is no class are left out
"""
import math
from types import SimpleNamespace

import torch

own = False

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5


def _group(name, op, x, dtype, images, positions, width, groups, act="silu", affine=True, gap=0):
    return {"name": name, "kind": "group", "op": op, "x": x, "dtype": dtype, "images": images, "positions": positions,
            "width": width, "groups": groups, "act": act, "affine": affine, "gap": gap}


def _class(name, op, dtype, rows, width, classes, bias=False, ignored=0.0, gap=0):
    return {"name": name, "kind": "class", "op": op, "dtype": dtype, "rows": rows, "width": width,
            "classes": classes, "bias": bias, "ignored": ignored, "gap": gap}


def _distill(name, op, dtype, rows, width, classes, top, tau=2.0, bias=False, ignored=0.0, gap=0):
    return {"name": name, "kind": "distill", "op": op, "dtype": dtype, "rows": rows, "width": width,
            "classes": classes, "top": top, "tau": tau, "bias": bias, "ignored": ignored, "gap": gap}


def listed():
    return [
        # One image through the last norm of the five-layer stack, as a server answers a request: 8x8 pixels of 64
        # channels of 8x8 capsules, a group for each two of them.  Latency counts.
        _group("group_fwd_one", "fwd", "bf16", "bf16", 1, 64, 4096, 32),
        # In the middle of the stack: 64 images of 16x16 pixels, the layer's fp32 result made the next one's bf16.
        _group("group_fwd_stack", "fwd", "fp32", "bf16", 64, 256, 4096, 32),
        # Benchmark configuration 2: 32x32 pixels, 32 channels of 3x3x3 capsules, each a group of 27 columns.
        _group("group_fwd_3d", "fwd", "fp32", "fp32", 64, 1024, 864, 32),
        # The way back through the stack's norm, everything in bf16.
        _group("group_bwd_stack", "bwd", "bf16", "bf16", 64, 256, 4096, 32),
        # 16x16 capsules, 64 channels, 32x32 pixels (benchmark configuration 5) of 16 images: groups of half a million values.
        _group("group_bwd_large", "bwd", "fp16", "fp16", 16, 1024, 16384, 32),
        # One feature vector of 64 channels of 8x8 capsules scored against many classes, as a server does.
        _class("class_fwd_one", "fwd", "bf16", 1, 4096, 50000),
        # The head of a training step: a long batch, a quarter of whose rows carry no target.
        _class("class_fwd_large", "fwd", "bf16", 8192, 4096, 131072, ignored=0.25),
        # A small classifier in fp32: the 864 values of a pixel of configuration 2, a thousand classes and one, with bias.
        _class("class_bwd_fp32", "bwd", "fp32", 1000, 864, 1001, bias=True),
        # The way back of a training step's head over an odd number of classes.
        _class("class_bwd_large", "bwd", "bf16", 8192, 2048, 100003),
        # A batch learning from 64 logits of a teacher for each row.
        _distill("distill_fwd_many", "fwd", "bf16", 4096, 2048, 65536, 64, ignored=0.1),
        # A short batch in fp16, an odd number of rows, few teacher's logits.
        _distill("distill_bwd_short", "bwd", "fp16", 509, 1024, 10007, 8, bias=True),
        # The way back of a batch learning from 64 logits for each row.
        _distill("distill_bwd_many", "bwd", "bf16", 4096, 2048, 65536, 64, ignored=0.1),
    ]


def draw(rng):
    """One more case.  Group norms: 1 to 256 images of 1 to 1024 positions, 8 to 16384 columns in 1 to 64 groups, every
    type, direction and activation.  Heads: 1 to 16384 rows of 16 to 8192 values, 10 to 131072 classes, 1 to 128
    teacher's logits, every type and direction."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if rng.random() < 0.4:
        groups = rng.choice([1, 2, 4, 8, 10, 16, 32, 64])
        columns = rng.choice([8, 16, 27, 30, 64, 64, 128, 256])
        columns *= rng.choice([k for k in (1, 1, 2, 3, 4, 8) if k * columns * groups <= 16384])
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        width, positions = groups * columns, log_int(1, 1024)
        images = max(1, min(log_int(1, 256), int(2.5e8 / (width * positions))))
        case = _group("", rng.choice(["fwd", "bwd"]), rng.choice(["fp32", dtype]), dtype, images, positions, width,
                      groups, rng.choice(["linear", "sigmoid", "silu", "silu"]), rng.random() < 0.8,
                      rng.choice([0, 0, 0, 8, 5]))
    else:
        dtype = rng.choice(["bf16", "fp16", "bf16", "fp16", "fp32"])
        rows, classes = log_int(1, 16384), log_int(10, 131072)
        width = log_int(2, 1024) * 8 + rng.choice([0, 0, 0, 0, 1, 3])
        op = rng.choice(["fwd", "bwd"])
        most = (8e12 if op == "fwd" else 3e12) * (0.25 if dtype == "fp32" else 1.0)
        rows = max(1, min(rows, int(most / (2.0 * width * classes))))
        more = dict(bias=rng.random() < 0.4, ignored=rng.choice([0.0, 0.0, 0.1, 0.5]), gap=rng.choice([0, 0, 0, 8, 5]))
        if rng.random() < 0.5:
            case = _class("", op, dtype, rows, width, classes, **more)
        else:
            case = _distill("", op, dtype, rows, width, classes, min(classes, log_int(1, 128)),
                            rng.choice([1.0, 2.0, 4.0]), **more)
    del case["name"]
    return case


# --------------------------------------------------------------------------------------- inputs
def _gapped(t, gap):
    """The same values in rows that lie apart."""
    if not gap:
        return t
    wide = torch.zeros((*t.shape[:-1], t.shape[-1] + gap), dtype=t.dtype, device=t.device)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def _group_inputs(case, gen):
    c = SimpleNamespace(**case)
    shape = (c.images, c.positions, c.width)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # a layer's result: columns differ in mean, images and groups in scale
    x = normal(*shape).mul_(normal(c.images, 1, c.groups).mul_(0.5).exp_().repeat_interleave(c.width // c.groups, 2))
    x.add_(normal(c.width).mul_(0.5))
    s = SimpleNamespace(x=_gapped(x.to(TORCH[c.x]), c.gap), weight=None, bias=None)
    del x
    if c.affine:
        s.weight, s.bias = normal(c.width).mul_(0.1).add_(1.0), normal(c.width).mul_(0.1)
    if c.op == "bwd":
        s.dy = _gapped(normal(*shape).mul_(0.1).to(TORCH[c.dtype]), c.gap)
        # the statistics that the way forward kept
        g = s.x.reshape(c.images, c.positions, c.groups, -1).double()
        mean = g.mean((1, 3))
        s.mean = mean.float()
        s.rstd = ((g - mean[:, None, :, None]).square().mean((1, 3)) + EPS).rsqrt().float()
    return s


def _head_inputs(case, gen):
    c = SimpleNamespace(**case)
    dtype = TORCH[c.dtype]

    def integers(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=gen, device="cuda")

    weight = torch.randn((c.classes, c.width), generator=gen, device="cuda").mul_(2.0 * c.width ** -0.5)
    x = torch.randn((c.rows, c.width), generator=gen, device="cuda")
    first = integers(0, c.classes, c.rows)
    # a network that has learnt something: rows lean towards their class, some much, some little
    x.add_(weight[first] * torch.rand((c.rows, 1), generator=gen, device="cuda").mul_(2.0))
    s = SimpleNamespace(x=_gapped(x.to(dtype), c.gap), weight=_gapped(weight.to(dtype), c.gap), bias=None)
    if c.bias:
        s.bias = torch.randn(c.classes, generator=gen, device="cuda").mul_(0.5)
    # rows without a target come in runs (a batch's padding)
    left = (torch.arange(c.rows, device="cuda") * 8 // max(1, c.rows) * 0.125 + 0.125 * torch.rand(
        c.rows, generator=gen, device="cuda")) < c.ignored
    if c.kind == "class":
        s.targets = torch.where(left, torch.full_like(first, -1), first)
    else:
        steps = integers(1, max(2, c.classes // c.top + 1), c.rows, c.top)
        steps[:, 0] = 0
        index = (first[:, None] + steps.cumsum(1)) % c.classes
        count = torch.where(torch.rand(c.rows, generator=gen, device="cuda") < 0.1,
                            integers(0, c.top + 1, c.rows), torch.full_like(first, c.top))
        gone = left[:, None] | (torch.arange(c.top, device="cuda") >= count[:, None])
        s.index = torch.where(gone, torch.full_like(index, -1), index)
        s.logits = torch.randn((c.rows, c.top), generator=gen, device="cuda").mul_(2.0).sort(1, descending=True)[0]
    if c.op == "bwd":
        s.dloss = torch.rand(c.rows, generator=gen, device="cuda").add_(0.5).div_(c.rows)
        # what the way forward kept, in 64 bits and some rows at a time
        kept = []
        wide = s.weight.double()
        for at in range(0, c.rows, 2048):
            z = s.x[at:at + 2048].double() @ wide.T
            z = (z if s.bias is None else z + s.bias.double()) / (c.tau if c.kind == "distill" else 1.0)
            lse = torch.logsumexp(z, 1)
            pick = s.targets[at:at + 2048, None] if c.kind == "class" else s.index[at:at + 2048]
            kept.append((lse, (z.gather(1, pick.clamp(min=0)) - lse[:, None]).masked_fill(pick < 0, 0.0)))
        lse, logq = (torch.cat([k[j] for k in kept]) for j in range(2))
        empty = s.targets < 0 if c.kind == "class" else (s.index < 0).all(1)
        s.lse = lse.masked_fill(empty, 0.0).float()
        if c.kind == "class":
            s.loss = -logq[:, 0].float()
        else:
            s.logq = logq.float()
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = (_group_inputs if case["kind"] == "group" else _head_inputs)(case, gen)
    s.case = case
    if own:
        from paper_2104_02621_amd import capscaps as cc
        s.cc = cc
    return s


# --------------------------------------------------------------------------------------- plain forms
def _act(kind, a):
    if kind == "linear":
        return a, torch.ones_like(a)
    q = 1.0 / (1.0 + torch.exp(-a))
    if kind == "sigmoid":
        return q, q * (1.0 - q)
    return a * q, q * (1.0 + a * (1.0 - q))


def _plain_group(s, c):
    x = s.x.float().reshape(c.images, c.positions, c.groups, -1)
    weight, bias = (None if t is None else t.view(c.groups, -1) for t in (s.weight, s.bias))
    if c.op == "fwd":
        mean = x.mean((1, 3), keepdim=True)
        x = x - mean
        rstd = 1.0 / (x.square().mean((1, 3), keepdim=True) + EPS).sqrt()
        x = x * rstd
        if c.affine:
            x = x * weight + bias
        return {"y": _act(c.act, x)[0].view(s.x.shape).to(TORCH[c.dtype]), "mean": mean.view(c.images, c.groups),
                "rstd": rstd.view(c.images, c.groups)}
    rstd = s.rstd[:, None, :, None]
    x = (x - s.mean[:, None, :, None]) * rstd
    d = s.dy.float().reshape(x.shape) * _act(c.act, x * weight + bias if c.affine else x)[1]
    got = {"dweight": None, "dbias": None}
    if c.affine:
        got = {"dweight": (d * x).sum((0, 1)).view(-1), "dbias": d.sum((0, 1)).view(-1)}
        d = d * weight
    d = rstd * (d - d.mean((1, 3), keepdim=True) - x * (d * x).mean((1, 3), keepdim=True))
    return {"dx": d.view(s.x.shape).to(TORCH[c.dtype]), **got}


def _plain_head(s, c):
    x, weight = s.x.float(), s.weight.float()
    z = x @ weight.T
    if c.bias:
        z = z + s.bias
    tau = 1.0
    if c.kind == "distill":
        tau = c.tau
        z = z / tau
        keep = s.index >= 0
        pick = s.index.clamp(min=0)
        teacher = torch.where(keep, s.logits / tau, torch.full_like(s.logits, -math.inf))
        top = teacher.amax(1, keepdim=True)
        e = torch.exp(teacher - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = e.sum(1, keepdim=True).clamp(min=1e-30)
        t = e / total
        logt = torch.where(keep, teacher - top - total.log(), torch.zeros_like(teacher))
        row = keep.any(1)
    else:
        row = s.targets >= 0
        keep, pick = row[:, None], s.targets.clamp(min=0)[:, None]
        t, logt = keep.float(), torch.zeros_like(z[:, :1])
    if c.op == "fwd":
        top = z.amax(1, keepdim=True)
        lse = top + torch.exp(z - top).sum(1, keepdim=True).log()
        logq = torch.where(keep, z.gather(1, pick) - lse, torch.zeros_like(t))
        lse = torch.where(row, lse[:, 0], torch.zeros_like(lse[:, 0]))
        loss = (tau * tau) * (t * (logt - logq)).sum(1)
        return {"loss": loss, "lse": lse, **({"logq": logq} if c.kind == "distill" else {})}
    g = torch.exp(z - s.lse[:, None])
    g.scatter_add_(1, pick, -t)
    g *= torch.where(row, s.dloss * tau, torch.zeros_like(s.dloss))[:, None]
    g = torch.where(row[:, None], g, torch.zeros_like(g))
    dtype = TORCH[c.dtype]
    return {"dx": (g @ weight).to(dtype), "dweight": (g.T @ x).to(dtype), "dbias": g.sum(0) if c.bias else None}


# --------------------------------------------------------------------------------------- the library's calls
def _library(s, c):
    cc = s.cc
    if c.kind == "group":
        same = dict(weight=s.weight, bias=s.bias, act=c.act)
        if c.op == "fwd":
            r = cc.group_norm_fwd(s.x, c.groups, dtype=TORCH[c.dtype], eps=EPS, save=True, **same)
            return {"y": r.y, "mean": r.mean, "rstd": r.rstd}
        r = cc.group_norm_bwd(s.x, c.groups, s.mean, s.rstd, s.dy, **same)
        return {"dx": r.dx, "dweight": r.dweight, "dbias": r.dbias}
    if c.kind == "class":
        if c.op == "fwd":
            r = cc.class_loss_fwd(s.x, s.weight, s.targets, bias=s.bias)
            return {"loss": r.loss, "lse": r.lse}
        r = cc.class_loss_bwd(s.x, s.weight, s.targets, s.loss, s.lse, s.dloss, bias=s.bias)
    else:
        same = dict(bias=s.bias, temperature=c.tau)
        if c.op == "fwd":
            r = cc.distill_loss_fwd(s.x, s.weight, s.index, s.logits, **same)
            return {"loss": r.loss, "lse": r.lse, "logq": r.logq}
        r = cc.distill_loss_bwd(s.x, s.weight, s.index, s.logits, s.lse, s.logq, s.dloss, **same)
    return {"dx": r.dx, "dweight": r.dweight, "dbias": r.dbias}


def run(s):
    c = SimpleNamespace(**s.case)
    if own:
        return _library(s, c)
    return (_plain_group if c.kind == "group" else _plain_head)(s, c)


# --------------------------------------------------------------------------------------- bytes and operations
def work(case):
    c = SimpleNamespace(**case)
    if c.kind == "group":
        n, layer, stats = c.images * c.positions * c.width, SIZE[c.dtype], 8 * c.images * c.groups
        if c.op == "fwd":
            return {"bytes": n * (SIZE[c.x] + layer) + stats + 8 * c.width * c.affine, "flops": n * 12}
        return {"bytes": n * (SIZE[c.x] + 2 * layer) + stats + 16 * c.width * c.affine, "flops": n * 24}
    size, rows = SIZE[c.dtype], c.rows * (1.0 - c.ignored)
    product = 2.0 * rows * c.width * c.classes
    top = 12 * c.rows * c.top if c.kind == "distill" else 8 * c.rows
    inputs = size * c.width * (rows + c.classes) + top + 4 * c.classes * c.bias
    if c.op == "fwd":
        kept = 4 * c.rows * c.top if c.kind == "distill" else 0
        return {"bytes": inputs + 8 * c.rows + kept, "flops": product}
    kept = 4 * c.rows * (2 + (c.top if c.kind == "distill" else 1))
    outputs = size * c.width * (c.rows + c.classes) + 4 * c.classes * c.bias
    return {"bytes": inputs + kept + outputs, "flops": 3 * product}


# --------------------------------------------------------------------------------------- in 64 bits
def _exact_group(s, c):
    """The norm as a function of x, weight and bias, image by image; its gradients by differentiating that function."""
    grad = c.op == "bwd"

    def leaf(t):
        return None if t is None else t.double().requires_grad_(grad)

    weight, bias = leaf(s.weight), leaf(s.bias)
    parts, sums = [], [0.0, 0.0]
    for i in range(c.images):
        x = leaf(s.x[i].contiguous())
        cols = x.view(c.positions, c.groups, -1).transpose(0, 1).reshape(c.groups, -1)
        var, mean = torch.var_mean(cols, dim=1, unbiased=False)
        a = torch.nn.functional.group_norm(x.T[None], c.groups, weight, bias, EPS)[0].T
        y = {"linear": lambda: a, "sigmoid": lambda: torch.sigmoid(a), "silu": lambda: a * torch.sigmoid(a)}[c.act]()
        if not grad:
            parts.append((y, mean, torch.rsqrt(var + EPS)))
            continue
        got = torch.autograd.grad(y, [x] + ([weight, bias] if c.affine else []), s.dy[i].double())
        parts.append(got[:1])
        sums = [total + g for total, g in zip(sums, got[1:])]
    whole = [torch.stack([p[j] for p in parts]) for j in range(len(parts[0]))]
    if grad:
        return {"dx": whole[0], "dweight": sums[0] if c.affine else None, "dbias": sums[1] if c.affine else None}
    return {"y": whole[0], "mean": whole[1], "rstd": whole[2]}


def _exact_rows(s, c, at, upto, weight, bias):
    """Loss and what is kept of some rows, as a function of x, weight and bias."""
    x = s.x[at:upto].double()
    if c.op == "bwd":
        x = x.requires_grad_()
    z = torch.nn.functional.linear(x, weight, bias)
    if c.kind == "class":
        target = s.targets[at:upto]
        logp = torch.log_softmax(z, 1)
        loss = torch.nn.functional.nll_loss(logp, target, ignore_index=-1, reduction="none")
        return x, loss, torch.logsumexp(z, 1) * (target >= 0), None
    index = s.index[at:upto]
    there = index >= 0
    some = there.any(1)
    logq = torch.log_softmax(z / c.tau, 1).gather(1, index.clamp(min=0))
    # (rows without entries: any finite values, which count nothing)
    teacher = (s.logits[at:upto].double() / c.tau).masked_fill(~there & some[:, None], -math.inf)
    logt = torch.log_softmax(teacher, 1).masked_fill(~there, 0.0)
    share = torch.softmax(teacher, 1).masked_fill(~there, 0.0)
    loss = c.tau ** 2 * (share * (logt - logq)).sum(1)
    return x, loss, torch.logsumexp(z / c.tau, 1) * some, logq.masked_fill(~there, 0.0)


def _exact_head(s, c):
    grad = c.op == "bwd"
    weight = s.weight.double().requires_grad_(grad)
    bias = None if s.bias is None else s.bias.double().requires_grad_(grad)
    parts, sums = [], [0.0, 0.0]
    step = max(256, min(c.rows, int(2e8 / c.classes)))
    for at in range(0, c.rows, step):
        x, loss, lse, logq = _exact_rows(s, c, at, at + step, weight, bias)
        if not grad:
            parts.append((loss, lse, logq))
            continue
        got = torch.autograd.grad(loss, [x, weight] + ([] if bias is None else [bias]), s.dloss[at:at + step].double())
        parts.append(got[:1])
        sums = [total + g for total, g in zip(sums, got[1:])]
    whole = [None if parts[0][j] is None else torch.cat([p[j] for p in parts]) for j in range(len(parts[0]))]
    if grad:
        return {"dx": whole[0], "dweight": sums[0], "dbias": None if bias is None else sums[1]}
    return {"loss": whole[0], "lse": whole[1], **({"logq": whole[2]} if c.kind == "distill" else {})}


def exact(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c = SimpleNamespace(**case)
    with torch.set_grad_enabled(c.op == "bwd"):
        if c.kind == "group":
            return _exact_group(_group_inputs(case, gen), c)
        with torch.no_grad():
            s = _head_inputs(case, gen)
        return _exact_head(s, c)
