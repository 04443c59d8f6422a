"""GPU parity of the gradient norm and of AdamW (32- and 8-bit moments) over lists of tensors: sizes from nothing to
past 32 bits, odd addresses, gradients of each type, copies, clipping, skipped steps, infinities and NaN."""
import numpy as np
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc
from tests import adamw_ref as ref

pytestmark = pytest.mark.gpu

FP32, BF16, FP16 = torch.float32, torch.bfloat16, torch.float16
U = 2.0 ** -24
LR, B1, B2, EPS = 1e-2, 0.9, 0.99, 1e-8


def control(scale=1.0, skip=0, step=1):
    c = torch.tensor([0.0, scale, 0.0, 0.0])
    c[2:].view(torch.int32).copy_(torch.tensor([skip, step], dtype=torch.int32))
    return c.cuda()


def state_of(c):
    c = c.cpu()
    return float(c[0]), float(c[1]), int(c[2:].view(torch.int32)[0]), int(c[2:].view(torch.int32)[1])


def at(t, shift):
    """`t` on the GPU, `shift` values into its allocation."""
    if not shift:
        return t.cuda()
    buf = torch.empty(t.numel() + shift, dtype=t.dtype, device="cuda")
    buf[shift:].copy_(t)
    return buf[shift:]


# ---------------------------------------------------------------------------------------- gradient norm
@pytest.mark.parametrize("sizes", [[1], [255, 0, 256, 257], [16384], [16385, 3], [100000, 1, 7, 40000], [5] * 300,
                                   [3_000_001]])
@pytest.mark.parametrize("dtype", [FP32, BF16, FP16])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_and_clipping(sizes, dtype, shift):
    rng = torch.Generator().manual_seed(sum(sizes))
    host = [torch.randn(n, generator=rng).to(dtype) for n in sizes]
    grads = [at(g, shift) for g in host]
    total = 0.5 * np.sqrt(sum(float((g.double() ** 2).sum()) for g in host))
    for most in (None, 0.25 * total, 4 * total):
        norm, scale, skip, step = state_of(cc.grad_norm(grads, max_norm=most, grad_scale=0.5))
        # fp64 sums (half a unit of fp32 after them), one rounding of the norm, two of the scale
        assert abs(norm - total) <= 2 * U * total
        want = 0.5 * min(1.0, (most or np.inf) / total)
        assert abs(scale - want) <= 4 * U * want
        assert (skip, step) == (0, 1)
    a, b = (cc.grad_norm(grads) for _ in range(2))
    assert torch.equal(a, b)


def test_norm_of_large_and_small_values():
    big = torch.full((1000,), 1e30, device="cuda")      # squares pass the largest float
    norm, scale, skip, _ = state_of(cc.grad_norm([big], max_norm=1.0))
    assert abs(norm - 1e30 * np.sqrt(1000)) <= 4 * U * norm and skip == 0
    assert abs(scale - 1 / norm) <= 8 * U / norm
    small = torch.full((1000,), 1e-30, device="cuda")
    norm, scale, skip, _ = state_of(cc.grad_norm([small], max_norm=1.0))
    assert abs(norm - 1e-30 * np.sqrt(1000)) <= 4 * U * norm and scale == 1.0
    assert state_of(cc.grad_norm([torch.zeros(5, device="cuda")], max_norm=1.0)) == (0.0, 1.0, 0, 1)
    c = torch.zeros(4, device="cuda")
    assert state_of(cc.grad_norm([], control=c)) == (0.0, 1.0, 0, 1)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", [0, 77, 20000])
def test_a_norm_that_is_not_finite_skips_the_step(bad, where):
    g = torch.ones(20001, device="cuda")
    c = torch.zeros(4, device="cuda")
    cc.grad_norm([g], max_norm=1.0, control=c)
    g[where] = bad
    cc.grad_norm([g], max_norm=1.0, control=c)
    norm, scale, skip, step = state_of(c)
    assert not np.isfinite(norm) and scale == 0.0 and skip == 1 and step == 1
    g[where] = 1.0
    assert state_of(cc.grad_norm([g], max_norm=1.0, control=c))[2:] == (0, 2)


# ---------------------------------------------------------------------------------------- AdamW
def tensors(sizes, rng, dtype=FP32, shift=0):
    """Parameters, gradients and decays; every fourth block of 256 gradients is zero."""
    params, grads = [], []
    for n in sizes:
        params.append(at(torch.randn(n, generator=rng) * 0.1, shift))
        g = torch.randn(n, generator=rng) * torch.exp(2 * torch.randn(n, generator=rng)) * 0.01
        g[(torch.arange(n) // 256) % 4 == 3] = 0.0
        grads.append(at(g.to(dtype), shift))
    return params, grads, [0.1 if n > 300 else 0.0 for n in sizes]


SIZES = [[1], [0, 5, 0], [255, 256, 257], [2047, 2048, 2049], [4096, 8192, 100], [70001], [300] * 100]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,copy,shift", [(FP32, None, 0), (FP32, BF16, 1), (BF16, FP16, 0), (FP16, BF16, 3)],
                         ids=["f32", "f32-off1-bf16", "bf16-f16", "f16-off3-bf16"])
def test_three_steps(sizes, bits, dtype, copy, shift):
    rng = torch.Generator().manual_seed(sum(sizes) + bits)
    params, grads, decay = tensors(sizes, rng, dtype, shift)
    copies = None if copy is None else [at(torch.zeros(n, dtype=copy), shift) for n in sizes]
    opt = cc.AdamW(params, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=decay, state_bits=bits, copies=copies, seed=99)
    if bits == 8 and shift:   # codes at odd addresses
        state = [[at(t.cpu(), shift) for t in s] for s in (opt.m, opt.v, opt.m_exp, opt.v_exp)]
        opt = cc.AdamW(params, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=decay, state_bits=8, copies=copies,
                       seed=99, state=state)
    # the reference goes on from the kernel's own parameters, so that only one step's rounding counts
    m, v = ([np.zeros(n, dtype=np.float32) for n in sizes] for _ in range(2))
    for t in range(1, 4):
        before = [p.cpu().numpy().copy() for p in params]
        opt.step(grads)
        for k, n in enumerate(sizes):
            p, m[k], v[k] = ref.step32(before[k], grads[k].float().cpu().numpy(), m[k], v[k], t, 1.0, LR, B1, B2, EPS, decay[k])
            got = params[k].cpu().numpy().astype(np.float64)
            # p: its product with 1 - lr * decay and the sum; the step: m and v exact, eight roundings and the bias corrections'
            move = np.abs(p - before[k] * (1 - LR * decay[k]))
            assert (np.abs(got - p) <= 3 * U * np.abs(before[k]) + 16 * U * move + 1e-40).all(), (k, n, t)
            if copies is not None:
                assert torch.equal(copies[k], params[k].to(copy)), (k, n, t)
            if bits == 32:
                assert np.array_equal(opt.m[k].cpu().numpy(), m[k]) and np.array_equal(opt.v[k].cpu().numpy(), v[k])
                continue
            rm, rv = ref.random16(0, n, 99, t, k)
            for name, x, r, codes, exps in (("m", m, rm, opt.m, opt.m_exp), ("v", v, rv, opt.v, opt.v_exp)):
                want, e = ref.encode(x[k], r, name == "m")
                assert np.array_equal(exps[k].cpu().numpy(), e), (name, k, n, t)
                assert np.array_equal(codes[k].cpu().numpy(), want), (name, k, n, t)
                x[k] = ref.decode(want, e, name == "m").astype(np.float32)
        if bits == 8:
            for got, want in zip(opt.state_values(), (m, v)):
                for a, b in zip(got, want):
                    assert a.dtype == BF16 and np.array_equal(a.float().cpu().numpy(), b)


@pytest.mark.parametrize("bits", [32, 8])
def test_control_gives_scale_step_and_skip(bits):
    rng = torch.Generator().manual_seed(4)
    params, grads, decay = tensors([513, 40], rng)
    copies = [p.to(BF16) for p in params]
    opt = cc.AdamW(params, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=decay, state_bits=bits, copies=copies)
    held = [t.clone() for t in params + copies + opt.m + opt.v]
    opt.step(grads, control=control(0.5, skip=1, step=3))
    opt.step(grads, control=control(0.5, skip=0, step=0))    # no step counted yet: nothing to correct the moments with
    for a, b in zip(held, params + copies + opt.m + opt.v):
        assert torch.equal(a, b)
    before = params[0].cpu().numpy().copy()
    opt.step(grads, control=control(0.37, step=7))
    p, m, v = ref.step32(before, grads[0].cpu().numpy(), np.zeros(513), np.zeros(513), 7, np.float32(0.37), LR, B1, B2, EPS, decay[0])
    # (the bias corrections are computed in fp32 here: expm1 to 2 ulp of 7 log(beta))
    move = np.abs(p - before * (1 - LR * decay[0]))
    assert (np.abs(params[0].cpu().numpy() - p) <= 3 * U * np.abs(before) + 32 * U * move + 1e-40).all()
    if bits == 8:
        want, e = ref.encode(m, ref.random16(0, 513, 0, 7, 0)[0], True)
        assert np.array_equal(opt.m[0].cpu().numpy(), want) and np.array_equal(opt.m_exp[0].cpu().numpy(), e)


def test_gradient_norm_then_step_as_a_training_loop_has_them():
    rng = torch.Generator().manual_seed(5)
    params, grads, decay = tensors([5000, 300, 27], rng)
    opt = cc.AdamW(params, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=decay)
    c = torch.zeros(4, device="cuda")
    m, v = ([np.zeros(p.numel()) for p in params] for _ in range(2))
    for t in range(1, 4):
        before = [p.cpu().numpy().copy() for p in params]
        cc.grad_norm(grads, max_norm=0.1, control=c)
        opt.step(grads, control=c)
        norm, scale, skip, step = state_of(c)
        assert (skip, step) == (0, t) and 0 < scale < 1
        for k in range(3):
            p, m[k], v[k] = ref.step32(before[k], grads[k].cpu().numpy(), m[k], v[k], t, np.float32(scale), LR, B1, B2, EPS, decay[k])
            move = np.abs(p - before[k] * (1 - LR * decay[k]))
            assert (np.abs(params[k].cpu().numpy() - p) <= 3 * U * np.abs(before[k]) + 32 * U * move + 1e-40).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_gradients_that_are_not_finite_stay_visible(bits, bad):
    """Without a control nothing is skipped: the value turns NaN, in 8 bits the moments of its block of 256."""
    p = torch.ones(1000, device="cuda")
    opt = cc.AdamW([p], state_bits=bits)
    g = torch.full((1000,), 0.1, device="cuda")
    g[300] = bad
    opt.step([g])
    assert torch.isnan(p[300]) and torch.isfinite(p[:300]).all() and torch.isfinite(p[301:]).all()
    m = opt.state_values()[0][0].float()
    if bits == 8:
        assert torch.isnan(m[256:512]).all() and torch.isfinite(m[:256]).all() and torch.isfinite(m[512:]).all()
        assert opt.m_exp[0].tolist()[1] == 255
    else:
        assert not torch.isfinite(m[300]) and torch.isfinite(m[:300]).all() and torch.isfinite(m[301:]).all()


def test_8_bit_moments_of_extreme_values():
    """The largest and smallest gradients, alone and next to each other in a block: codes by the definition."""
    g = torch.tensor([0.0, 1e-45, 1e-38, 1.2e-38, 1e-30, -1e-22, 1e-19, 1e-10, 1.0, -3.0, 1e10, 1e18, 3e38, -0.0])
    for part in (g, g[:3], g[:5], g[:8], g[3:4], g[11:12], g[12:13] * 0.9):
        n = len(part)
        p = torch.zeros(n, device="cuda")
        opt = cc.AdamW([p], lr=LR, betas=(B1, B2), state_bits=8, seed=3)
        opt.step([part.cuda()])
        _, m, v = ref.step32(np.zeros(n), part.numpy(), np.zeros(n), np.zeros(n), 1, 1.0, LR, B1, B2, EPS, 0.0)
        rm, rv = ref.random16(0, n, 3, 1, 0)
        want, e = ref.encode(m, rm, True)
        assert np.array_equal(opt.m_exp[0].cpu().numpy(), e)
        assert np.array_equal(opt.m[0].cpu().numpy() & 127, want & 127)
        want, e = ref.encode(v, rv, False)
        assert np.array_equal(opt.v_exp[0].cpu().numpy(), e)
        if e[0] != 255:
            assert np.array_equal(opt.v[0].cpu().numpy(), want)


def test_rounding_at_random_keeps_the_expected_moments():
    """A variance that is to fall by a factor of four over 3000 steps of a thousandth: rounded to nearest it would not
    move at all.  65536 values, whose errors are independent to within their codes' spread (about 0.2): their mean is off by about 0.001."""
    n, steps, b2 = 65536, 3000, 0.999
    p = torch.zeros(n, device="cuda")
    opt = cc.AdamW([p], lr=0.0, betas=(0.9, b2), state_bits=8, seed=17)
    gen = torch.Generator(device="cuda").manual_seed(8)
    g = torch.randn(n, generator=gen, device="cuda").sign_()
    opt.step([2 * g])                         # v = 0.001 * 4
    start = float(opt.state_values()[1][0].double().mean())
    assert abs(start - 0.004) <= 0.02 * 0.004
    for _ in range(steps):
        opt.step([g])
    want = 0.004 * b2 ** steps + (1 - b2 ** steps)
    m, v = (t[0].double() for t in opt.state_values())
    assert abs(float(v.mean()) - want) <= 0.02 * want
    assert abs(float((m * g).mean()) - 1.0) <= 0.02


def test_steps_repeat_bit_for_bit_and_seeds_differ():
    def run(seed, stream=None):
        rng = torch.Generator().manual_seed(6)
        params, grads, decay = tensors([70001, 50], rng)
        opt = cc.AdamW(params, state_bits=8, seed=seed, weight_decay=decay)
        for _ in range(3):
            opt.step(grads)
        return params + opt.m + opt.v
    a, b, c = run(1), run(1), run(2)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert not all(torch.equal(x, y) for x, y in zip(a, c))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_saved_state_goes_on_as_it_was(bits):
    def run(stop):
        rng = torch.Generator().manual_seed(12)
        params, grads, _ = tensors([3000, 41], rng)
        opt = cc.AdamW(params, state_bits=bits, seed=4)
        for k in range(4):
            if k == stop:
                state = [[t.clone() for t in s] for s in (opt.m, opt.v, opt.m_exp, opt.v_exp)[:4 if bits == 8 else 2]]
                opt = cc.AdamW(params, state_bits=bits, seed=4, state=state, steps=opt.steps)
            opt.step(grads)
        return params + opt.m + opt.v
    for a, b in zip(run(None), run(2)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_tensor_past_32_bits(bits):
    """2^31 + 300 values: the last ones against the reference."""
    n, tail = (1 << 31) + 300, 812          # (whole blocks of 256 from n - 812 on)
    p = torch.zeros(n, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    rng = torch.Generator().manual_seed(7)
    p[-tail:] = torch.randn(tail, generator=rng).cuda()
    g[-tail:] = torch.randn(tail, generator=rng).to(BF16).cuda()
    before = p[-tail:].cpu().numpy()
    opt = cc.AdamW([p], lr=LR, betas=(B1, B2), eps=EPS, state_bits=bits, seed=5)
    norm = state_of(cc.grad_norm([g]))[0]
    want = float(g[-tail:].double().square().sum().sqrt())
    assert abs(norm - want) <= 2 * U * want
    opt.step([g])
    zero = np.zeros(tail)
    want, m, v = ref.step32(before, g[-tail:].float().cpu().numpy(), zero, zero, 1, 1.0, LR, B1, B2, EPS, 0.0)
    assert (np.abs(p[-tail:].cpu().numpy() - want) <= 3 * U * np.abs(before) + 16 * U * LR + 1e-40).all()
    assert (n - tail) % 256 == 0
    if bits == 8:
        rm, rv = ref.random16(n - tail, tail, 5, 1, 0)
        for x, r, codes, signed in ((m, rm, opt.m[0], True), (v, rv, opt.v[0], False)):
            assert np.array_equal(codes[-tail:].cpu().numpy(), ref.encode(x, r, signed)[0])
    else:
        assert np.array_equal(opt.m[0][-tail:].cpu().numpy(), m)


def test_a_captured_training_step_replays_as_it_ran():
    """Norms, gradient norm and AdamW in one graph: steps are counted on the device, so each replay is the next step."""
    rng = torch.Generator().manual_seed(9)
    x, b, dh = (torch.randn((64, 200), generator=rng).cuda() for _ in range(3))

    def program():
        w = [torch.ones(200, device="cuda"), torch.full((200,), 0.5, device="cuda")]
        opt, c = cc.AdamW(w, lr=0.05, state_bits=8), torch.zeros(4, device="cuda")

        def step():
            r = cc.block_norm_fwd(x, b, pre_weight=w[0], post_weight=w[1], save=True)
            g = cc.block_norm_bwd(r.y, b, r.rstd_pre, r.rstd_post, dh, None, pre_weight=w[0], post_weight=w[1])
            grads = [g.dpre_weight, g.dpost_weight]
            cc.grad_norm(grads, max_norm=0.5, control=c)
            opt.step(grads, control=c)
        return w, c, step

    w0, c0, eager = program()
    w1, c1, step = program()
    held = [t.clone() for t in w1]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, w1))   # captured, not run
    for k in range(5):
        eager()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c0, c1) and state_of(c1)[3] == k + 1
        assert all(torch.equal(a, b) for a, b in zip(w0, w1)), k
