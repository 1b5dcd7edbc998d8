"""The AdamW step of many tensors, states in 32 bits and in 8, against plain implementations in 64 bits, and its refusals."""
import ctypes as C

import pytest
import torch

from paper_2511_20426_amd import binding as B

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}        # a rounding, relative: half a step
U = 2.0 ** -24
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "f32": torch.float32}
HYPER = dict(lr=3e-3, betas=(0.9, 0.98), eps=1e-7, weight_decay=0.1)


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _packed(gen, sizes, dtype, scale=1.0):
    """tensors one behind the other in one piece of memory, so that most begin at an odd place; the piece"""
    flat = (torch.randn(sum(sizes), generator=gen, dtype=torch.float64) * scale).to(dtype).to(DEV)
    ends = torch.tensor(sizes).cumsum(0).tolist()
    return [flat[e - n:e] for e, n in zip(ends, sizes)], flat


def _values(c, a, v):
    """codes of whole blocks and their scales, in 64 bits"""
    c, a = c.double().view(-1, 256), a.double()[:, None]
    return ((c / 255) ** 4 * a if v else c.sign() * (c / 127) ** 2 * a).flatten()


def _check_codes(got, x, scales, v):
    """got: the codes of whole blocks of x.  A code is the whole number next to 255 (x / a)^(1/4) or 127 (|x| / a)^(1/2); computed here, in 64 bits, that is
    off by a few roundings of 2^-53 of a number up to 255, less than 1e-12, which decides next to a border: gradients of 26.875 and 107.5 at a first step
    give m = 2.6875 (1 - 2^-53) beside a = 10.75, 63.5 but for 2^-54 of it: 63, and rounded ahead of the border 64."""
    x = x.view(-1, 256)
    most = x.abs().amax(1)
    # the scale is that in fp32, of half a step at most; next to the middle of two either (9.2700846195220965 of fp32's 9.27008438 and 9.27008533)
    a = scales
    assert ((a.double() - most).abs() <= U * (1 + 1e-9) * most + 1e-45).all()
    got, part = got.double().view(-1, 256), x.abs() / torch.where(a > 0, a, 1).double()[:, None]
    t = 255 * part.sqrt().sqrt() if v else 127 * part.sqrt()
    if v:
        t = torch.where((x > 0) & (t < 1), 1.0, t)
    t = t.clamp(max=255 if v else 127)                               # (a scale is rounded, and may be less than what it stands for)
    wrong = torch.nonzero((((got.abs() - t * (a > 0)[:, None]).abs() > 0.5 + 1e-12) | (got * x < 0)).flatten())[:, 0]
    assert wrong.numel() == 0, [(k.item(), got.flatten()[k].item(), x.flatten()[k].item().hex(), a[k // 256].item().hex()) for k in wrong[:9]]


def _check_step(opt, params, grads, states, before, steps, scale=1.0, lr=None):
    """states: m, v (64 bits) of each tensor ahead of the step, whole blocks; before: the parameters then"""
    (b1, b2), eps, wd, lr = opt.betas, opt.eps, opt.weight_decay, opt.lr if lr is None else lr
    for i, (p, g) in enumerate(zip(params, grads)):
        at, n = opt.offsets[i], p.numel()
        room = opt.offsets[i + 1] - at
        m0, v0 = states[i]
        if g is None:
            m, v = m0, v0
        else:
            gd = torch.zeros(room, dtype=torch.float64)
            gd[:n] = g.double().cpu().flatten() * scale
            m, v = b1 * m0 + (1 - b1) * gd, b2 * v0 + (1 - b2) * gd * gd
        got_m, got_v = opt.m[at:at + room].cpu(), opt.v[at:at + room].cpu()
        if opt.state_bits == 32:
            # factors, products and the sum are rounded once each
            assert ((got_m.double() - m).abs() <= 4 * U * (m0.abs() + m.abs())).all(), i
            assert ((got_v.double() - v).abs() <= 6 * U * v + 1e-44).all(), i
        else:
            for got, x, scales, isv in ((got_m, m, opt.m_scale, False), (got_v, v, opt.v_scale, True)):
                if g is not None:
                    _check_codes(got, x, scales[at // 256:(at + room) // 256].cpu(), isv)
        if n == 0:
            continue
        old, new = before[i].double().cpu().flatten(), p.double().cpu().flatten()
        if g is None:
            assert torch.equal(old, new)
            continue
        t = steps[i]
        denom = (v[:n] / (1 - b2 ** t)).sqrt() + eps
        move = lr / (1 - b1 ** t) * m[:n] / denom
        ref = (1 - lr * wd) * old - move
        # m as above, v under a root, rate, quotient and their product: less than 16 roundings
        way = 16 * U * move.abs() + lr / (1 - b1 ** t) / denom * 4 * U * m0[:n].abs() + 3 * U * (old.abs() + ref.abs())
        assert ((new - ref).abs() <= HALF[p.dtype] * (ref.abs() + way) + way + 1e-45).all(), i


def _states(opt):
    m, v = opt.state_values()
    if opt.state_bits == 8:
        dm, dv = _values(opt.m.cpu(), opt.m_scale.cpu(), False), _values(opt.v.cpu(), opt.v_scale.cpu(), True)
        assert ((m.double().cpu() - dm).abs() <= U * 1.01 * dm.abs() + 1e-45).all() and ((v.double().cpu() - dv).abs() <= U * 1.01 * dv + 1e-45).all()
    else:
        dm, dv = m.double().cpu(), v.double().cpu()
    return [(dm[a:b].clone(), dv[a:b].clone()) for a, b in zip(opt.offsets, opt.offsets[1:])]


SIZES = [[1], [3, 0, 255, 256, 257], [511, 512, 513, 5], [40000, 1, 777], [(i * 37) % 600 + (i % 9 > 0) for i in range(710)], [3000001]]


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("param", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_steps(which, bits, param, grad):
    """Tensors at odd places, some without a gradient at some steps, gradients of very different sizes and zeros"""
    from paper_2511_20426_amd.optim import AdamW
    sizes, gen = SIZES[which], _gen(which)
    params, flat = _packed(gen, sizes, T[param], 0.1)
    opt = AdamW(params, state_bits=bits, **HYPER)
    steps = [0] * len(sizes)
    for trip in range(3):
        grads, _ = _packed(gen, sizes, T[grad], 10.0 ** (-3 * trip))
        grads = [g * torch.exp(2 * torch.randn(g.shape, generator=gen).to(DEV)).to(g.dtype) for g in grads]
        if len(sizes) > 1:
            grads[-1][::3] = 0
            grads[trip] = None
        before, states = [p.clone() for p in params], _states(opt)
        scale = (1.0, 0.37, 1e-4)[trip]
        opt.step(grads, grad_scale=scale)
        steps = [s + (g is not None and g.numel() > 0) for s, g in zip(steps, grads)]
        assert opt.steps.tolist() == steps
        _check_step(opt, params, grads, states, before, steps, scale)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_shapes_and_copies_and_a_schedule(bits):
    from paper_2511_20426_amd.optim import AdamW
    gen = _gen(9)
    params = [torch.randn(s, generator=gen).to(DEV) for s in ((5, 7), (2, 3, 129), ())]
    copies = [torch.full(params[0].shape, 7.0, dtype=torch.bfloat16, device=DEV), None, torch.zeros((), dtype=torch.bfloat16, device=DEV)]
    opt = AdamW(params, state_bits=bits, copies=copies, **HYPER)
    for t in (1, 2):
        grads = [torch.randn(p.shape, generator=gen).to(DEV) for p in params]
        before, states = [p.clone() for p in params], _states(opt)
        opt.lr = 0.01 / t
        opt.step(grads)
        _check_step(opt, params, grads, states, before, [t] * 3)
        assert all(c is None or torch.equal(c, p.bfloat16()) for c, p in zip(copies, params))


@pytest.mark.gpu
def test_large_tensor_of_several_units_to_a_wave():
    """More than 4096 workgroups' worth of values: checked as the rest, on the device"""
    from paper_2511_20426_amd.optim import AdamW
    n = 4096 * 4 * 512 * 2 + 300
    p, g = torch.full((n,), 0.5, device=DEV), torch.linspace(-1, 1, n, device=DEV)
    opt = AdamW([p], state_bits=8, **HYPER)
    opt.step([g])
    m = (1 - 0.9) * g.double()
    whole = torch.zeros(opt.offsets[1], dtype=torch.float64, device=DEV)
    whole[:n] = m
    _check_codes(opt.m, whole, opt.m_scale, False)
    denom = ((1 - 0.98) * g.double() ** 2 / (1 - 0.98)).sqrt() + HYPER["eps"]
    ref = (1 - HYPER["lr"] * HYPER["weight_decay"]) * 0.5 - HYPER["lr"] / (1 - 0.9) * m / denom
    assert ((p.double() - ref).abs() <= 24 * U * (0.5 + HYPER["lr"])).all()
    assert opt.steps.tolist() == [1]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_count_on(bits):
    """A captured step, replayed between eager ones with other work and waits between them, gives what as many eager steps give"""
    from paper_2511_20426_amd.optim import AdamW
    gen, sizes = _gen(3), [700, 31, 5000]
    runs = []
    for _ in range(2):
        params, flat = _packed(_gen(3), sizes, torch.float32)
        runs.append((params, flat, AdamW(params, state_bits=bits, **HYPER)))
    grads, gflat = _packed(gen, sizes, torch.bfloat16)
    (p0, f0, a), (p1, f1, b) = runs
    a.step(grads)
    b.step(grads)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step(grads)
    assert a.steps.tolist() == [1] * 3                               # a capture runs nothing
    for trip in range(4):
        gflat.copy_(torch.randn(sum(sizes), generator=gen))
        graph.replay()
        b.step(grads)
        torch.cuda.synchronize()
        assert torch.equal(f0, f1) and torch.equal(a.m, b.m) and torch.equal(a.v, b.v) and a.steps.tolist() == b.steps.tolist() == [2 + 2 * trip] * 3
        a.step(grads)
        b.step(grads)
        assert torch.equal(f0, f1)


@pytest.mark.gpu
def test_gradients_that_are_not_finite():
    """32 bits: the values themselves; 8 bits: all that share the scale.  Others stay what they would be."""
    from paper_2511_20426_amd.optim import AdamW
    for bits in (32, 8):
        for bad in (float("inf"), float("nan"), 1e30):
            g = torch.ones(1024, device=DEV)
            p, q = torch.zeros(1024, device=DEV), torch.zeros(1024, device=DEV)
            one, other = AdamW([p], state_bits=bits), AdamW([q], state_bits=bits)
            other.step([g])
            g = g.clone()
            g[300] = bad
            one.step([g])
            (m, v), (m1, v1) = one.state_values(), other.state_values()
            hit = torch.zeros(1024, dtype=torch.bool, device=DEV)
            hit[256:512] = bits == 8
            hit[300] = True
            for x, y in ((m, m1), (v, v1)):
                assert torch.equal(x[~hit], y[~hit])
            assert not v[hit].isfinite().any()
            near = torch.arange(1024, device=DEV) != 300
            assert torch.equal(p[near], q[near])


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_small_and_zero_gradients(bits):
    """Zeros leave states of zero; gradients whose squares pass below fp32 move nothing far: m / (sqrt(v) + eps) with v of zero"""
    from paper_2511_20426_amd.optim import AdamW
    p, g = torch.ones(600, device=DEV), torch.zeros(600, device=DEV)
    opt = AdamW([p], lr=1.0, eps=1e-8, weight_decay=0.0, state_bits=bits)
    opt.step([g])
    m, v = opt.state_values()
    assert (p == 1).all() and (m == 0).all() and (v == 0).all()
    g += 1e-26
    opt.step([g])
    assert ((p - 1).abs() < 1e-15).all() and p.isfinite().all()
    for _ in range(3):
        opt.step([0 * g])
    assert p.isfinite().all()


@pytest.mark.gpu
def test_other_stream_and_state_loaded():
    from paper_2511_20426_amd.optim import AdamW
    gen, sizes = _gen(4), [300, 1000]
    params, flat = _packed(gen, sizes, torch.bfloat16)
    grads, _ = _packed(gen, sizes, torch.bfloat16)
    opt = AdamW(params, state_bits=8, **HYPER)
    for _ in range(3):
        opt.step(grads)
    twin = flat.clone()
    again = AdamW([twin[:300], twin[300:]], state_bits=8, **HYPER)
    again.load_state(opt.m, opt.v, opt.steps.tolist(), opt.m_scale, opt.v_scale)
    opt.step(grads)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again.step(grads)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(flat, twin) and torch.equal(opt.m, again.m) and torch.equal(opt.v, again.v) and again.steps.tolist() == [4, 4]


@pytest.mark.gpu
def test_arguments_refused_on_device():
    from paper_2511_20426_amd.optim import AdamW
    p = torch.zeros((6, 16), device=DEV)
    for bad in (lambda: AdamW([]), lambda: AdamW([p.half()]), lambda: AdamW([p.t()]), lambda: AdamW([p, p]), lambda: AdamW([p[:4], p[2:]]),
                lambda: AdamW([p], state_bits=16), lambda: AdamW([p.cpu()]), lambda: AdamW([p], copies=[p]), lambda: AdamW([p], copies=[]),
                lambda: AdamW([p.bfloat16()], copies=[p.bfloat16()])):
        with pytest.raises(AssertionError):
            bad()
    opt = AdamW([p])
    for bad in ([], [p, p], [p.half()], [p[:5]], [p.cpu()], [torch.zeros((16, 6), device=DEV).t()]):
        with pytest.raises(AssertionError):
            opt.step(bad)
    for name, bad in (("lr", -1.0), ("lr", float("nan")), ("betas", (1.0, 0.9)), ("betas", (0.9, -0.1)), ("eps", 0.0), ("weight_decay", -1.0)):
        keep = getattr(opt, name)
        setattr(opt, name, bad)
        with pytest.raises(B.CascadeAttnError):
            opt.step([p.clone()])
        setattr(opt, name, keep)
    assert (p == 0).all() and opt.steps.tolist() == [0]


def test_arguments_refused():
    """On the host, before anything is launched"""
    at = 4096

    def call(n=1, bits=8, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, scale=1.0, table=at, **change):
        t = (B.ca_adamw_tensor * 1)()
        for name, value in {**dict(param=at, grad=at, copy=0, m=at, v=at, m_scale=at, v_scale=at, step=at, n=10, param_dtype=B.CA_F32,
                                   grad_dtype=B.CA_BF16), **change}.items():
            setattr(t[0], name, value)
        B.layer_adamw(t, table, n, bits, lr, b1, b2, eps, wd, scale)

    for change, code in ((dict(n=-1), B.CA_EINVAL), (dict(table=0), B.CA_EINVAL), (dict(table=at + 8), B.CA_EINVAL), (dict(bits=16), B.CA_EINVAL), (dict(lr=-1.0), B.CA_EINVAL), (dict(lr=1e39), B.CA_EINVAL), (dict(b1=1.0), B.CA_EINVAL),
                         (dict(b2=float("nan")), B.CA_EINVAL), (dict(eps=0.0), B.CA_EINVAL), (dict(eps=1e-60), B.CA_EINVAL), (dict(wd=-0.1), B.CA_EINVAL),
                         (dict(scale=float("inf")), B.CA_EINVAL), (dict(param=0), B.CA_EINVAL), (dict(param=at + 2), B.CA_EINVAL), (dict(grad=at + 1), B.CA_EINVAL),
                         (dict(m=0), B.CA_EINVAL), (dict(m=at + 8), B.CA_EINVAL), (dict(v=at + 4), B.CA_EINVAL), (dict(m_scale=0), B.CA_EINVAL),
                         (dict(v_scale=at + 2), B.CA_EINVAL), (dict(step=0), B.CA_EINVAL), (dict(step=at + 8), B.CA_EINVAL), (dict(copy=at + 1), B.CA_EINVAL),
                         (dict(copy=at, param_dtype=B.CA_BF16), B.CA_EINVAL), (dict(param_dtype=5), B.CA_EINVAL), (dict(grad_dtype=-1), B.CA_EINVAL)):
        if "n" in change:
            change = {"n": change["n"]}
        with pytest.raises(B.CascadeAttnError) as e:
            call(**change)
        assert e.value.code == code, change
    t = (B.ca_adamw_tensor * 1)()
    t[0].n = -5
    with pytest.raises(B.CascadeAttnError):
        B.layer_adamw(t, at, 1, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0)
    t[0].n = 2 ** 41
    with pytest.raises(B.CascadeAttnError) as e:
        B.layer_adamw(t, at, 1, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0)
    assert e.value.code == B.CA_EUNSUPPORTED
    t[0].n = 7                                                       # without a gradient nothing is done
    B.layer_adamw(t, at, 1, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0)
    B.layer_adamw(None, 0, 0, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0)
    for bad in ((0, at, at, at, at, at, 256), (at, at + 8, at, at, at, at, 256), (at, at, 0, at, at, at, 256), (at, at, at, at, at + 4, at, 256),
                (at, at, at, at, at, at, 255), (at, at, at, at, at, at, -256)):
        with pytest.raises(B.CascadeAttnError):
            B.layer_adamw_values(*bad)
    B.layer_adamw_values(0, 0, 0, 0, 0, 0, 0)
    assert C.sizeof(B.ca_adamw_tensor) == 80
