"""Performance cases of the operators that train and serve a stack of capsule layers: the norms around a block
with its gate and residual, the norm of all gradients, and the AdamW step over many tensors.

`run` computes them in plain torch operations in 32 bits, or, with `own`, through the library's entry points.
`listed()` holds fixed cases; `draw(rng)` makes more of the ranges they stand for; `exact` computes the same from
the definitions in 64 bits.

Notation.  Block norm: rows of `width` values, x the residual stream, b the block's output,
    y = residual_scale x + branch_scale act(gate) (b / rms(b)) post_weight,      h = (y / rms(y)) pre_weight.
AdamW in 8 bits: 256 consecutive values of a moment share an exponent byte E.  The first moment's code is a sign
bit and a magnitude c, 0 or (c + 8 (E - 15)) << 20 as the bits of an fp32 value; the second moment's code c is 0
or (c + 8 (E - 31)) << 20.  Both are rounded up or down at random, by the bits of `mix`.
"""
import math
from types import SimpleNamespace

import torch

own = False

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6
LR, BETA1, BETA2, ADAM_EPS = 1e-3, 0.9, 0.999, 1e-8
MASK = 0xFFFFFFFF

# kernel tensors of the five-layer stack of 8x8 capsules, of benchmark configuration 5 (16x16 capsules, 64 to 64
# channels, 3x3 window), of the small layers, and norm weights of their widths
STACK = [294912, 589824, 1179648, 2359296, 2621440]
LARGE = 9437184


def _norm(name, op, dtype, stream, branch, rows, width, gate="none", act="linear", post=True, scales=(1.0, 1.0),
          gap=0):
    return {"name": name, "kind": "norm", "op": op, "dtype": dtype, "stream": stream, "branch": branch,
            "rows": rows, "width": width, "gate": gate, "act": act, "post": post, "residual_scale": scales[0],
            "branch_scale": scales[1], "gap": gap}


def _tensors(name, kind, sizes, **more):
    return {"name": name, "kind": kind, "sizes": ",".join(map(str, sizes)), **more}


def listed():
    return [
        # One image through the last block of the five-layer stack, as a server answers a request: 8x8 pixels
        # of 64 channels of 8x8 capsules.  Latency counts.
        _norm("norm_fwd_one", "fwd", "bf16", "bf16", "bf16", 64, 4096, "shared"),
        # Benchmark configuration 2: 64 images of 32x32 pixels, 32 channels of 3x3x3 capsules, in fp32.
        _norm("norm_fwd_3d", "fwd", "fp32", "fp32", "fp32", 65536, 864, "shared", scales=(1.0, 0.5)),
        # Every 8x8 capsule of benchmark configuration 3 normalised by itself, with a gate for each value.
        _norm("norm_fwd_caps", "fwd", "bf16", "bf16", "bf16", 128 * 28 * 28 * 64, 64, "full", "sigmoid"),
        # The way back through a block in the middle of the stack: 64 images of 16x16 pixels, 64 channels of 8x8
        # capsules, residual stream and convolution result in fp32.
        _norm("norm_bwd_stack", "bwd", "bf16", "fp32", "fp32", 16384, 4096, "shared"),
        # 3x3x3 capsules by themselves: rows of 27 values, which no vector load divides.
        _norm("norm_bwd_27", "bwd", "fp32", "fp32", "fp32", 64 * 32 * 32 * 32, 27, "full", "silu"),
        # 16x16 capsules, 64 channels (benchmark configuration 5) of 16 images: the widest rows and most bytes.
        _norm("norm_bwd_large", "bwd", "fp16", "fp16", "fp16", 16384, 16384, "shared", scales=(0.9, 1.0)),
        # The norm of all gradients of the five-layer stack, for clipping.
        _tensors("gradnorm_stack", "gradnorm", STACK + [2048, 2048, 4096, 4096]),
        # ... and of twelve layers of benchmark configuration 5.
        _tensors("gradnorm_large", "gradnorm", [LARGE] * 12 + [16384, 16384]),
        # The optimizer of a network of one small layer (benchmark configuration 1): a few thousand parameters.
        _tensors("adamw32_small", "adamw", [2304, 64, 64], bits=32, copy="none"),
        # Twelve layers of benchmark configuration 5, with the fp16 kernels that the next step reads.
        _tensors("adamw32_large", "adamw", [LARGE] * 12 + [16384, 16384], bits=32, copy="fp16"),
        # The five-layer stack and some odd vectors, moments in 8 bits, bf16 kernels for the next step.
        _tensors("adamw8_stack", "adamw", STACK + [2048, 2048, 4096, 4096, 600, 27, 1], bits=8, copy="bf16"),
        # Twelve layers of benchmark configuration 5 with moments in 8 bits.
        _tensors("adamw8_large", "adamw", [LARGE] * 12 + [16384, 16384], bits=8, copy="fp16"),
    ]


def draw(rng):
    """One more case: rows of 8 to 16384 values (4x4 to 16x16 capsules, alone or 1 to 64 channels together), 1 to 10
    million rows, every type, gate and direction; lists of 1 to 14 tensors of 1 to 10 million values."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if rng.random() < 0.5:
        caps = rng.choice([8, 16, 20, 27, 30, 64, 64, 128, 256])
        width = caps * rng.choice([1, 1, 3, 4, 10, 14, 16, 20, 32, 33, 64])
        dtype = rng.choice(["fp32", "bf16", "fp16"])
        stream, branch = rng.choice(["fp32", dtype]), rng.choice(["fp32", dtype])
        rows = log_int(1, 1 << 23)
        gate = rng.choice(["none", "shared", "full"])
        case = _norm("", rng.choice(["fwd", "bwd"]), dtype, stream, branch, rows, width, gate,
                     rng.choice(["linear", "sigmoid", "silu"]) if gate != "none" else "linear",
                     rng.random() < 0.8, (rng.choice([1.0, 0.9]), rng.choice([1.0, 0.5])),
                     rng.choice([0, 0, 0, 8, 5]))
        case["rows"] = max(1, min(rows, int(3e9 / (work(case)["bytes"] / rows))))
    else:
        top = log_int(1000, LARGE)
        sizes = [log_int(max(1, top // 100), top) for _ in range(rng.randint(1, 10))]
        sizes += [rng.choice([1, 27, 64, 600, 2048]) for _ in range(rng.randint(0, 4))]
        if rng.random() < 0.3:
            case = _tensors("", "gradnorm", sizes)
        else:
            case = _tensors("", "adamw", sizes, bits=rng.choice([8, 32]), copy=rng.choice(["none", "bf16", "fp16"]))
    del case["name"]
    return case


# --------------------------------------------------------------------------------------- inputs
def _sizes(case):
    return [int(s) for s in case["sizes"].split(",")]


def _norm_inputs(case, gen):
    c = SimpleNamespace(**case)
    layer, stream, branch = TORCH[c.dtype], TORCH[c.stream], TORCH[c.branch]

    def rows_of(dtype, sigma):
        # a capsule's scale differs from pixel to pixel
        x = torch.randn((c.rows, c.width), generator=gen, device="cuda")
        x.mul_(torch.randn((c.rows, 1), generator=gen, device="cuda").mul_(0.5).exp_().mul_(sigma))
        if not c.gap:
            return x.to(dtype)
        wide = torch.zeros((c.rows, c.width + c.gap), dtype=dtype, device="cuda")
        wide[:, :c.width] = x
        return wide[:, :c.width]

    def vector(mean, sigma):
        return torch.randn(c.width, generator=gen, device="cuda").mul_(sigma).add_(mean)

    s = SimpleNamespace(x=rows_of(stream, 1.0), b=rows_of(branch, 0.7), gate=None, wpre=vector(1.0, 0.1),
                        wpost=vector(1.0, 0.1) if c.post else None)
    if c.gate == "shared":
        s.gate = vector(0.5, 0.3)
    elif c.gate == "full":
        s.gate = rows_of(layer, 1.0)
    if c.op == "bwd":
        # x stands for the block's result y here; the statistics are those that the way forward kept
        s.dh, s.dy = rows_of(layer, 0.1), rows_of(stream, 0.1)
        s.rpre, s.rpost = (1.0 / (t.float().square().mean(1) + EPS).sqrt() for t in (s.x, s.b))
        if not c.post:
            s.rpost = None
    return s


def _codes(gen, n, top, low, high, sign):
    """Codes and exponents of a moment in 8 bits: magnitudes low .. high, exponents around `top`."""
    c = torch.randint(low, high, (n,), generator=gen, device="cuda", dtype=torch.uint8)
    if sign:
        c |= torch.randint(0, 2, (n,), generator=gen, device="cuda", dtype=torch.uint8) << 7
    e = torch.randint(top - 1, top + 2, ((n + 255) // 256,), generator=gen, device="cuda").to(torch.uint8)
    return c, e


def _tensor_inputs(case, gen, seed):
    s = SimpleNamespace(step=1 + seed % 997, seed=seed & 0xFFFF, grads=[], params=[], m=[], v=[], me=[], ve=[])
    s.copies = []
    for k, n in enumerate(_sizes(case)):
        scale = 10.0 ** -(2 + k % 3)  # layers differ in the size of their gradients
        g = torch.randn(n, generator=gen, device="cuda").mul_(scale)
        g[n // 2:n // 2 + n // 16] = 0.0  # channels that never fired
        s.grads.append(g)
        if case["kind"] == "gradnorm":
            continue
        s.params.append(torch.randn(n, generator=gen, device="cuda").mul_(0.05))
        if case["bits"] == 32:
            s.m.append(torch.randn(n, generator=gen, device="cuda").mul_(0.3 * scale))
            s.v.append(torch.rand(n, generator=gen, device="cuda").add_(0.5).mul_(scale * scale))
        else:
            exponent = 127 + math.floor(math.log2(scale))
            m, me = _codes(gen, n, exponent, 70, 128, True)
            v, ve = _codes(gen, n, 127 + 2 * (exponent - 127), 200, 256, False)
            for t in (m, v):
                t[n // 2:n // 2 + n // 16] = 0
            s.m.append(m), s.v.append(v), s.me.append(me), s.ve.append(ve)
        if case["copy"] != "none":
            s.copies.append(torch.empty(n, dtype=TORCH[case["copy"]], device="cuda"))
    if case["kind"] == "adamw":
        # what the norm of the gradients left: norm, scale, whether to skip the step, the step's number
        s.control = torch.tensor([2.7, 0.37, 0.0, 0.0], device="cuda")
        s.control[2:].view(torch.int32).copy_(torch.tensor([0, s.step], dtype=torch.int32))
        # matrices decay, vectors do not
        s.decay = [0.1 if n > 16384 else 0.0 for n in _sizes(case)]
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["kind"] == "norm":
        s = _norm_inputs(case, gen)
    else:
        s = _tensor_inputs(case, gen, seed)
    s.case = case
    if own:
        from paper_2104_02621_amd import capscaps as cc
        s.cc = cc
        if case["kind"] == "gradnorm":
            s.control = torch.zeros(4, device="cuda")
            s.norm, s.scale = s.control[0], s.control[1]
        elif case["kind"] == "adamw":  # the optimizer that a training program keeps
            s.opt = cc.AdamW(s.params, lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=s.decay,
                             state_bits=case["bits"], copies=s.copies or None, seed=s.seed,
                             state=(s.m, s.v, s.me, s.ve) if case["bits"] == 8 else (s.m, s.v))
            if case["bits"] == 8:
                s.values = [[torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in _sizes(case)]
                            for _ in range(2)]
    return s


# --------------------------------------------------------------------------------------- plain forms
def _act(kind, g):
    if kind == "linear":
        return g, torch.ones_like(g)
    q = 1.0 / (1.0 + torch.exp(-g))
    if kind == "sigmoid":
        return q, q * (1.0 - q)
    return g * q, q * (1.0 + g * (1.0 - q))


def _plain_norm_fwd(s, c):
    u = s.b.float()
    rpost = None
    if c.post:
        rpost = 1.0 / (u.square().mean(1, keepdim=True) + EPS).sqrt()
        u = u * rpost * s.wpost
    if s.gate is not None:
        u = u * _act(c.act, s.gate.float())[0]
    y = c.residual_scale * s.x.float() + c.branch_scale * u
    rpre = 1.0 / (y.square().mean(1, keepdim=True) + EPS).sqrt()
    h = y * rpre * s.wpre
    return {"y": y.to(TORCH[c.stream]), "h": h.to(TORCH[c.dtype]), "rpre": rpre[:, 0],
            "rpost": None if rpost is None else rpost[:, 0]}


def _plain_norm_bwd(s, c):
    dh, rpre = s.dh.float(), s.rpre[:, None]
    yh = s.x.float() * rpre
    n = dh * s.wpre
    d = s.dy.float() + rpre * (n - yh * (n * yh).mean(1, keepdim=True))
    got = {"dx": (c.residual_scale * d).to(TORCH[c.stream]), "dwpre": (dh * yh).sum(0), "dwpost": None, "dgate": None}
    d = c.branch_scale * d
    bh = s.b.float()
    if c.post:
        bh = bh * s.rpost[:, None]
    if s.gate is not None:
        a, slope = _act(c.act, s.gate.float())
        dg = d * (bh * s.wpost if c.post else bh) * slope
        got["dgate"] = dg.sum(0) if c.gate == "shared" else dg.to(TORCH[c.dtype])
        d = d * a
    if c.post:
        got["dwpost"] = (d * bh).sum(0)
        d = d * s.wpost
        d = s.rpost[:, None] * (d - bh * (d * bh).mean(1, keepdim=True))
    got["db"] = d.to(TORCH[c.dtype])
    return got


def _plain_gradnorm(s):
    norm = torch.stack([g.square().sum() for g in s.grads]).sum().sqrt()
    return {"norm": norm, "scale": torch.clamp(1.0 / norm, max=1.0)}


def mix(x):
    """The bits that decide how a moment's value is rounded, from a number of 32 bits (a tensor or an int)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & MASK
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & MASK
    return x ^ (x >> 16)


def _dither(n, seed, step, k):
    key = mix((seed + 0x9E3779B1 * k + 0x6A09E667 * mix(step)) & MASK)
    i = torch.arange(n, device="cuda", dtype=torch.int64)
    x = mix((i * 0x9E3779B1 + key) & MASK)
    return x & 0xFFFF, x >> 16


def _decode(code, e, below, sign):
    c = code.to(torch.int32)
    mag = c & 127 if sign else c
    e = e.to(torch.int32).repeat_interleave(256)[:len(c)]
    x = ((mag + 8 * (e - below)) << 20).view(torch.float32)
    x = torch.where(mag == 0, torch.zeros_like(x), x)
    x = torch.where(e == 255, torch.full_like(x, math.nan), x)
    return torch.where(c > 127, -x, x) if sign else x


def _encode(x, random, below, sign):
    """Codes and exponents of fp32 values; `random`: 16 bits for each."""
    n = len(x)
    bits = x.abs().view(torch.int32)
    top = torch.nn.functional.pad(bits, (0, -n % 256)).view(-1, 256).amax(1)
    e = ((top + 0xFFFFF) >> 23).clamp(below + 1, 254)
    e = torch.where(top >= 0x7F800000, torch.full_like(e, 255), e)
    c = ((bits.long() + (random << 4)) >> 20) - 8 * (e.long().repeat_interleave(256)[:n] - below)
    if sign:
        c = c.clamp(0, 127) | ((x < 0).long() << 7)
    else:
        c = torch.maximum(c.clamp(0, 255), (bits > 0).long())
    return c.to(torch.uint8), e.to(torch.uint8)


def _plain_adamw_one(s, k, bits):
    p, g, m, v = s.params[k], s.grads[k], s.m[k], s.v[k]
    bc1, bc2 = 1.0 - BETA1 ** s.step, 1.0 - BETA2 ** s.step
    go = s.control.view(torch.int32)[2] == 0
    if bits == 8:
        m, v = _decode(m, s.me[k], 15, True), _decode(v, s.ve[k], 31, False)
    g = g * s.control[1]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    new = p * (1.0 - LR * s.decay[k]) - (LR / bc1) * (m / (v.sqrt() / math.sqrt(bc2) + ADAM_EPS))
    p.copy_(torch.where(go, new, p))
    if s.copies:
        s.copies[k].copy_(p)
    if bits == 32:
        s.m[k].copy_(torch.where(go, m, s.m[k]))
        s.v[k].copy_(torch.where(go, v, s.v[k]))
        return s.m[k], s.v[k]
    rm, rv = _dither(len(p), s.seed, s.step, k)
    for new, old in zip(_encode(m, rm, 15, True) + _encode(v, rv, 31, False), (s.m[k], s.me[k], s.v[k], s.ve[k])):
        old.copy_(torch.where(go, new, old))
    # the values the codes stand for, all of which bfloat16 holds exactly
    return (_decode(s.m[k], s.me[k], 15, True).bfloat16(), _decode(s.v[k], s.ve[k], 31, False).bfloat16())


def _plain(s, case):
    c = SimpleNamespace(**case)
    if c.kind == "norm":
        return _plain_norm_fwd(s, c) if c.op == "fwd" else _plain_norm_bwd(s, c)
    if c.kind == "gradnorm":
        return _plain_gradnorm(s)
    moments = [_plain_adamw_one(s, k, c.bits) for k in range(len(s.params))]
    return {"p": s.params, "copy": s.copies, "m": [t[0] for t in moments], "v": [t[1] for t in moments]}


# --------------------------------------------------------------------------------------- the library's calls
def _library(s, case):
    cc = s.cc
    if case["kind"] == "gradnorm":
        cc.grad_norm(s.grads, max_norm=1.0, control=s.control)
        return {"norm": s.norm, "scale": s.scale}
    if case["kind"] == "adamw":
        s.opt.step(s.grads, control=s.control)
        if case["bits"] == 8:
            m, v = s.opt.state_values(out=s.values)
        else:
            m, v = s.m, s.v
        return {"p": s.params, "copy": s.copies, "m": m, "v": v}
    same = dict(pre_weight=s.wpre, post_weight=s.wpost, gate=s.gate, gate_act=case["act"], post_norm=case["post"],
                residual_scale=case["residual_scale"], branch_scale=case["branch_scale"])
    if case["op"] == "fwd":
        r = cc.block_norm_fwd(s.x, s.b, dtype=TORCH[case["dtype"]], eps=EPS, save=True, **same)
        return {"y": r.y, "h": r.h, "rpre": r.rstd_pre, "rpost": r.rstd_post}
    r = cc.block_norm_bwd(s.x, s.b, s.rpre, s.rpost, s.dh, s.dy, **same)
    return {"dx": r.dx, "dwpre": r.dpre_weight, "dwpost": r.dpost_weight, "dgate": r.dgate, "db": r.dbranch}


def run(s):
    return _library(s, s.case) if own else _plain(s, s.case)


# --------------------------------------------------------------------------------------- bytes and operations
def work(case):
    size = {"fp32": 4, "bf16": 2, "fp16": 2, "none": 0}
    if case["kind"] == "norm":
        n, w, layer = case["rows"] * case["width"], case["width"], size[case["dtype"]]
        stream, branch = size[case["stream"]], size[case["branch"]]
        full, vectors = case["gate"] == "full", 1 + case["post"] + (case["gate"] == "shared")
        stats = 4 * case["rows"] * (1 + case["post"])
        if case["op"] == "fwd":
            return {"bytes": n * (2 * stream + branch + layer + full * layer) + 4 * w * vectors + stats,
                    "flops": n * (6 + 4 * case["post"] + 2 * (case["gate"] != "none"))}
        return {"bytes": n * (3 * stream + branch + 2 * layer + 2 * full * layer) + 8 * w * vectors + stats,
                "flops": n * (14 + 10 * case["post"] + 5 * (case["gate"] != "none"))}
    n = sum(_sizes(case))
    if case["kind"] == "gradnorm":
        return {"bytes": 4 * n + 8, "flops": 2 * n}
    state = 16 if case["bits"] == 32 else 4 + 4 + sum(4 * ((k + 255) // 256) for k in _sizes(case)) / n
    return {"bytes": n * (12 + state + size[case["copy"]]), "flops": 16 * n}


# --------------------------------------------------------------------------------------- in 64 bits
def _exact_norm(s, c):
    """The block as a function of x, b, gate and weights; its gradients by differentiating that function."""
    def leaf(t):
        return None if t is None else t.double().requires_grad_(c.op == "bwd")

    def rms_norm(t, w):
        return t / torch.sqrt(torch.mean(t * t, dim=1, keepdim=True) + EPS) * w

    def squash(g):
        return {"linear": lambda: g, "sigmoid": lambda: torch.sigmoid(g), "silu": lambda: g * torch.sigmoid(g)}[c.act]()

    def rstd(t):
        return torch.rsqrt(torch.mean(t * t, dim=1) + EPS)

    x, b, gate, wpre, wpost = (leaf(t) for t in (s.x, s.b, s.gate, s.wpre, s.wpost))
    branch = rms_norm(b, wpost) if c.post else b
    if gate is not None:
        branch = branch * squash(gate)
    if c.op == "fwd":
        y = c.residual_scale * x + c.branch_scale * branch
        return {"y": y, "h": rms_norm(y, wpre), "rpre": rstd(y), "rpost": rstd(b) if c.post else None}
    # s.x is y: the gradient that reaches y is dy and what comes through h
    h = rms_norm(x, wpre)
    dyt, dwpre = torch.autograd.grad(h, (x, wpre), s.dh.double())
    dyt = dyt + s.dy.double()
    wanted = [t for t in (b, gate, wpost) if t is not None]
    found = iter(torch.autograd.grad(branch, wanted, c.branch_scale * dyt))
    db, dgate, dwpost = (None if t is None else next(found) for t in (b, gate, wpost))
    return {"dx": c.residual_scale * dyt, "dwpre": dwpre, "dwpost": dwpost, "dgate": dgate, "db": db}


def _moment(code, e, below, sign):
    """A moment's values from the fields of its codes."""
    code, e = code.long(), e.double().repeat_interleave(256)[:len(code)]
    mag = code % 128 if sign else code
    x = torch.exp2(e - 127 - below + mag // 8) * (1.0 + (mag % 8) / 8.0) * (mag > 0)
    return x * (1 - 2 * (code // 128)) if sign else x


def _rounded(x, random, below, sign):
    """`x` on the grid of its block's codes: up or down by whether the fraction and the random one reach 1."""
    n, a = len(x), x.abs()
    top = torch.nn.functional.pad(a, (0, -n % 256)).view(-1, 256).amax(1)
    e = torch.floor(torch.log2(top.clamp(min=1e-300)))
    e = torch.where(top / torch.exp2(e) > 1.875, e + 1, e).clamp(below + 1 - 127, 127)
    e = e.repeat_interleave(256)[:n]
    grid = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -126))) - 3)
    q = torch.floor(a / grid + random.double() / 65536) * grid
    q = torch.minimum(q, 1.875 * torch.exp2(e))
    least = 1.125 * torch.exp2(e - below)
    if sign:
        return torch.where(q < least, torch.zeros_like(q), q) * torch.sign(x)
    return torch.where(a >= 2.0 ** -149, torch.maximum(q, least), torch.zeros_like(q))


def _exact_adamw(s, k, bits):
    m, v, g = s.m[k], s.v[k], s.grads[k].double() * s.control[1].double()
    m, v = (_moment(m, s.me[k], 15, True), _moment(v, s.ve[k], 31, False)) if bits == 8 else (m.double(), v.double())
    m = BETA1 * m + (1.0 - BETA1) * g
    v = BETA2 * v + (1.0 - BETA2) * g * g
    mhat, vhat = m / (1.0 - BETA1 ** s.step), v / (1.0 - BETA2 ** s.step)
    p = s.params[k].double()
    p = p - LR * (mhat / (vhat.sqrt() + ADAM_EPS) + s.decay[k] * p)
    if bits == 8:
        rm, rv = _dither(len(p), s.seed, s.step, k)
        m, v = _rounded(m, rm, 15, True), _rounded(v, rv, 31, False)
    return p, m, v


def exact(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    c = SimpleNamespace(**case)
    if c.kind == "norm":
        with torch.set_grad_enabled(c.op == "bwd"):
            return _exact_norm(_norm_inputs(case, gen), c)
    s = _tensor_inputs(case, gen, seed)
    if c.kind == "gradnorm":
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s.grads))
        return {"norm": norm, "scale": min(1.0, 1.0 / norm)}
    new = [_exact_adamw(s, k, c.bits) for k in range(len(s.params))]
    p, m, v = ([t[j] for t in new] for j in range(3))
    return {"p": p, "copy": p if s.copies else [], "m": m, "v": v}
