"""Performance cases of the operators that a layer is adapted with: the norm of its input with its gradients, low-rank adapters beside a
projection with theirs, and the step of the optimizer.

A case is one pass through one of them, as a program built on the library makes it:

  norm          layer norm of a layer's rows; weight and bias may be those of the block in flight that a row belongs to (modulation by its timestep)
  norm_grad     the same in training: forward, then the gradients of x, weights and biases
  adapted       a projection with low-rank adapters of many requests at once: each row has an adapter of its own, or none
  adapted_grad  the same in training over frozen weights: forward, then the gradients of x and of the adapters
  adamw         an AdamW step over many tensors at once, states in 32 bits or in 8

Sizes are the Wan shapes of `workloads` (width 1536 and 5120, blocks of 3 x 30 x 52 tokens), those of the tests, and single tokens.

The definitions.  Norm of a row x of W values: y = w (x - mean) / sqrt(mean((x - mean)^2) + eps) + b.  Adapted projection:
y = x W' + s_g (x A_g') B_g' with g the row's adapter; adapter -1: y = x W'.  AdamW: m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2,
p = (1 - lr wd) p - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps).  States in 8 bits, in blocks of 256 consecutive values of a tensor with a
scale a (fp32) each, the largest magnitude: m stands for sign(c) a (c / 127)^2 with whole c, |c| = round(127 sqrt(|m| / a)); v for a (c / 255)^4,
c = round(255 (v / a)^(1/4)), at least 1 where v > 0.  The step itself goes by m and v before they are brought to 8 bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
BLOCK = 256                                                        # values to a scale; tensors' states begin at its multiples
HYPER = {"lr": 1e-3, "betas": (0.9, 0.999), "eps": 1e-8, "weight_decay": 0.01}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(kind, rows, width, groups=1, dtype="bf16"):
    return {"kind": kind, "rows": rows, "width": width, "groups": groups, "dtype": dtype}


def _adapted(kind, rows, width, n_out, adapters, rank, mixed):
    """mixed: every row has an adapter of its own; otherwise runs of rows have, as blocks in flight do"""
    return {"kind": kind, "rows": rows, "width": width, "n_out": n_out, "adapters": adapters, "rank": rank, "mixed": mixed}


def _adamw(tensors, most, bits, param="f32", grad="bf16", odd=False):
    """tensors of `most` values and, odd, every other one of fewer"""
    return {"kind": "adamw", "tensors": tensors, "most": most, "bits": bits, "param": param, "grad": grad, "odd": odd}


def listed():
    return [
        # one token's row at the 14B width: all latency
        dict(_norm("norm", 1, 5120), name="norm_token"),
        # five blocks in flight at the 14B width, each modulated by its timestep: memory traffic
        dict(_norm("norm", 23400, 5120, groups=5), name="norm_wan14b"),
        # gradients in fp32 of an odd number of rows of an odd width: a check beside a new model
        dict(_norm("norm_grad", 433, 129, dtype="f32"), name="norm_grad_f32"),
        # a training step on one block of the 1.3B model
        dict(_norm("norm_grad", 4680, 1536), name="norm_grad_wan1p3b"),
        # one token of a request with an adapter: the weights' way from memory
        dict(_adapted("adapted", 1, 5120, 5120, 8, 16, True), name="adapted_token"),
        # a few hundred tokens of many requests, odd sizes
        dict(_adapted("adapted", 257, 1024, 776, 6, 5, True), name="adapted_odd"),
        # the 14B QKV projection of five blocks with an adapter each
        dict(_adapted("adapted", 23400, 5120, 15360, 5, 32, False), name="adapted_wan14b_qkv"),
        # a training step of one adapter of the 1.3B QKV projection
        dict(_adapted("adapted_grad", 4680, 1536, 4608, 1, 32, False), name="adapted_grad_wan1p3b"),
        # the two matrices of one adapter: latency
        dict(_adamw(2, 16 * 1536, 32), name="adamw_adapter"),
        # the adapters of thirty layers' projections, masters in fp32
        dict(_adamw(120, 32 * 1536, 32), name="adamw_adapters"),
        # the gated feed-forward half of the 1.3B model, states in 8 bits
        dict(_adamw(3, 4096 * 1536, 8, param="bf16"), name="adamw8_wan1p3b"),
        # that of the 14B model
        dict(_adamw(3, 13824 * 5120, 8, param="bf16"), name="adamw8_wan14b"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "adapted", "adapted", "adapted_grad", "adamw", "adamw"])
    if kind in ("norm", "norm_grad"):
        groups = rng.choice([1, 1, 2, 3, 5])
        rows = groups * _log_int(rng, 1, 23400 // groups)
        width = rng.choice([rng.choice([128, 256, 512, 768, 1024, 1536, 2048, 4096, 5120]), _log_int(rng, 8, 5120)])
        return _norm(kind, rows, width, groups, rng.choice(["bf16", "bf16", "f32"]))
    if kind in ("adapted", "adapted_grad"):
        grads = kind == "adapted_grad"
        rows, width = _log_int(rng, 1, 4680 if grads else 23400), 128 * rng.choice([1, 2, 3, 5, 8, 12, 20, 32, 40])
        n_out = 128 * rng.choice([1, 2, 3, 6, 9, 12, 20, 36, 40])
        if not grads and rng.random() < 0.5:
            n_out = 8 * (2 * _log_int(rng, 8, 320) - 1)
        return _adapted(kind, rows, width, n_out, rng.choice([1, 2, 3, 5, 8]), rng.choice([1, 4, 8, 16, 24, 32, 64, 100, 128]), rng.random() < 0.5)
    tensors = rng.choice([1, 2, 3, 7, 20, 75, 130])
    return _adamw(tensors, _log_int(rng, 1, min(13824 * 5120, 120000000 // tensors)), rng.choice([8, 32]), rng.choice(["f32", "bf16"]),
                  rng.choice(["bf16", "f32"]), rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs

def _sizes(case):
    return [case["most"] if not case["odd"] or i % 2 == 0 else max(1, case["most"] * (i % 7 + 1) // 9) for i in range(case["tensors"])]


def _places(sizes):
    """of each value of the tensors, packed one behind the other, its place where each tensor begins at a multiple of BLOCK; and how many
    places there are"""
    n = torch.tensor(sizes, device=DEVICE)
    room = (n + BLOCK - 1) // BLOCK * BLOCK
    shift = (room.cumsum(0) - room) - (n.cumsum(0) - n)
    return torch.arange(sum(sizes), device=DEVICE) + torch.repeat_interleave(shift, n, output_size=sum(sizes)), sum(-(-k // BLOCK) * BLOCK for k in sizes)


def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dtype)

    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        m, w, g, dtype = case["rows"], case["width"], case["groups"], DTYPES[case["dtype"]]
        x = normal(m, w, dtype=torch.float32) * torch.exp(0.5 * normal(w, dtype=torch.float32)) + normal(w, scale=0.5, dtype=torch.float32)
        shape = (w,) if g == 1 else (g, w)
        s = {"x": x.to(dtype), "weight": 1 + normal(*shape, scale=0.2, dtype=torch.float32), "bias": normal(*shape, scale=0.2, dtype=torch.float32)}
        if kind == "norm_grad":
            s["dy"] = normal(m, w, dtype=dtype)
        return s
    if kind in ("adapted", "adapted_grad"):
        m, k, n, g, r = case["rows"], case["width"], case["n_out"], case["adapters"], case["rank"]
        s = {"x": normal(m, k), "w": normal(n, k, scale=k ** -0.5), "down": normal(g, r, k, scale=k ** -0.5), "up": normal(g, n, r, scale=0.3 * r ** -0.5),
             "scales": 0.5 + torch.rand(g, generator=gen, device=DEVICE)}
        if case["mixed"]:                                          # a sixth of the rows or so has none
            index = torch.randint(-1, max(g, 5), (m,), generator=gen, device=DEVICE)
            s["index"] = torch.where(index < g, index, index % g).to(torch.int32)
        else:
            s["index"] = (torch.arange(m, device=DEVICE) * g // m).to(torch.int32)
        if kind == "adapted_grad":
            s["dy"] = normal(m, n)
        return s
    sizes = _sizes(case)
    total = sum(sizes)
    at, room = _places(sizes)
    s = {"p": normal(total, scale=0.02, dtype=DTYPES[case["param"]])}
    s["g"] = (normal(total, scale=1e-3, dtype=torch.float32) * torch.exp(normal(total, dtype=torch.float32))).to(DTYPES[case["grad"]])
    # states of a training under way
    m = torch.zeros(room, device=DEVICE).index_copy_(0, at, normal(total, scale=5e-4, dtype=torch.float32))
    v = torch.zeros(room, device=DEVICE).index_copy_(0, at, torch.exp(normal(total, scale=1.5, dtype=torch.float32)) * 1e-6)
    s["at"], s["sizes"], s["step"] = at, sizes, 100
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
        return s
    m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
    s["m_scale"], s["v_scale"] = m.abs().amax(1), v.amax(1)
    s["m"] = torch.round(m.sign() * 127 * (m.abs() / s["m_scale"][:, None]).sqrt()).to(torch.int8)
    s["v"] = torch.round(255 * (v / s["v_scale"][:, None]) ** 0.25).clamp(min=1).mul(v > 0).to(torch.uint8)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "adapted_grad":
        s["w_t"] = s["w"].t().contiguous()                         # frozen: laid out once for the way back
    if kind == "adamw" and own:
        from paper_2511_20426_amd.optim import AdamW
        ends = torch.tensor(s["sizes"]).cumsum(0).tolist()
        params, s["grads"] = ([s[t][e - n:e] for e, n in zip(ends, s["sizes"])] for t in ("p", "g"))
        s["optimizer"] = AdamW(params, state_bits=case["bits"], **HYPER)
        scales = {"m_scale": s["m_scale"], "v_scale": s["v_scale"]} if case["bits"] == 8 else {}
        s["optimizer"].load_state(s["m"].view(-1), s["v"].view(-1), step=s["step"], **scales)
    elif own and kind == "norm":
        s["y"] = torch.empty_like(s["x"])
    elif own and kind in ("adapted", "adapted_grad"):
        from paper_2511_20426_amd.runner import Adapters
        s["adapters"] = Adapters.from_weights(s["down"], s["up"], s["scales"])
        s["y"] = torch.empty((case["rows"], case["n_out"]), dtype=torch.bfloat16, device=DEVICE)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _by_row(t, rows):
    """of a weight [width] as it is, of weights [groups, width] that of each row"""
    return t if t.dim() == 1 else t.repeat_interleave(rows // t.shape[0], 0)


def _plain_norm(s):
    case = s["case"]
    m, dtype = case["rows"], s["x"].dtype
    w, b = _by_row(s["weight"], m), _by_row(s["bias"], m)
    x = s["x"].float()
    off = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((off * off).mean(-1, keepdim=True) + EPS)
    normed = off * r
    y = (normed * w + b).to(dtype)
    if case["kind"] == "norm":
        return y
    dy = s["dy"].float()
    dn = dy * w
    dx = r * (dn - dn.mean(-1, keepdim=True) - normed * (dn * normed).mean(-1, keepdim=True))
    groups = (case["groups"], m // case["groups"], case["width"])
    dw, db = ((t.view(groups).sum(1, dtype=torch.float64).float().view(s["weight"].shape)) for t in (dy * normed, dy))
    return {"y": y, "dx": dx.to(dtype), "dweight": dw, "dbias": db}


def _plain_adapted(s):
    case = s["case"]
    g, r, n, k = case["adapters"], case["rank"], case["n_out"], case["width"]
    x, w = s["x"].float(), s["w"].float()
    down, up = s["down"].float().reshape(g * r, k), s["up"].float().permute(0, 2, 1).reshape(g * r, n)
    # what of [rows, adapters x rank] belongs to a row's own adapter
    mine = (s["index"][:, None] == torch.arange(g, device=DEVICE)) * s["scales"]
    mine = mine.repeat_interleave(r, 1)
    t = (x @ down.T) * mine
    y = (x @ w.T + t @ up).to(torch.bfloat16)
    if case["kind"] == "adapted":
        return y
    dy = s["dy"].float()
    u = (dy @ up.T) * mine
    d_up = (t.T @ dy).view(g, r, n).permute(0, 2, 1)
    grads = {"dx": dy @ w + u @ down, "d_down": (u.T @ x).view(g, r, k), "d_up": d_up}
    return {"y": y, **{name: v.to(torch.bfloat16).contiguous() for name, v in grads.items()}}


def _values(s):
    """m and v of states in 8 bits, in 64"""
    c = s["m"].double()
    m = c * c.abs() / 127 ** 2 * s["m_scale"].double()[:, None]
    v = (s["v"].double() / 255).square().square() * s["v_scale"].double()[:, None]
    return m.view(-1), v.view(-1)


def _to_8_bits(s, m, v):
    """in 64 bits, for values next to a border between two codes"""
    m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
    s["m_scale"], s["v_scale"] = m.abs().amax(1).float(), v.amax(1).float()
    a, b = ((t.double()[:, None]) for t in (s["m_scale"], s["v_scale"]))
    codes = torch.round(127 * (m.abs() / torch.where(a > 0, a, 1)).sqrt()).clamp(max=127)
    s["m"] = (torch.sign(m) * codes * (a > 0)).to(torch.int8)
    codes = torch.round(255 * (v / torch.where(b > 0, b, 1)).sqrt().sqrt()).clamp(min=1, max=255)
    s["v"] = (codes * (v > 0) * (b > 0)).to(torch.uint8)


def _plain_adamw(s):
    bits, at, (b1, b2) = s["case"]["bits"], s["at"], HYPER["betas"]
    s["step"] += 1
    g = s["g"].float() if bits == 32 else s["g"].double()
    m_all, v_all = (s["m"], s["v"]) if bits == 32 else _values(s)
    m = b1 * m_all[at] + (1 - b1) * g
    v = b2 * v_all[at] + (1 - b2) * (g * g)
    m_all[at], v_all[at] = m, v
    m, v, p = m.float(), v.float(), s["p"].float()
    p = (1 - HYPER["lr"] * HYPER["weight_decay"]) * p - HYPER["lr"] / (1 - b1 ** s["step"]) * m / ((v / (1 - b2 ** s["step"])).sqrt() + HYPER["eps"])
    s["p"].copy_(p)                                                # rounded once
    if bits == 8:
        _to_8_bits(s, m_all, v_all)
        m_all, v_all = (t.float() for t in _values(s))
    return {"p": s["p"], "m": m_all, "v": v_all}


def _plain(s):
    kind = s["case"]["kind"]
    return _plain_norm(s) if kind in ("norm", "norm_grad") else _plain_adamw(s) if kind == "adamw" else _plain_adapted(s)


# ------------------------------------------------------------------------------------------------ the operators

def run(s):
    if not own:
        return _plain(s)
    kind = s["case"]["kind"]
    if kind == "adamw":
        s["optimizer"].step(s["grads"])
        m, v = s["optimizer"].state_values()                       # 32 bits: the states themselves; 8 bits: what they stand for
        return {"p": s["p"], "m": m, "v": v}
    from paper_2511_20426_amd import runner
    if kind == "norm":
        return runner.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, out=s["y"])
    if kind == "norm_grad":
        y = runner.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
        dx, dw, db = runner.layer_norm_backward(s["dy"], s["x"], s["weight"], s["bias"], eps=EPS)
        return {"y": y, "dx": dx, "dweight": dw, "dbias": db}
    if kind == "adapted":
        return runner.linear_adapted(s["x"], s["w"], s["adapters"], s["index"], out=s["y"])
    y, saved = runner.linear_adapted_train(s["x"], s["w"], s["adapters"], s["index"], out=s["y"])
    dx, d_down, d_up = runner.linear_adapted_backward(s["dy"], s["x"], s["w_t"], s["adapters"], s["index"], saved)
    return {"y": y, "dx": dx, "d_down": d_down, "d_up": d_up}


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        one, weights = case["rows"] * case["width"] * DTYPES[case["dtype"]].itemsize, 4 * case["groups"] * case["width"]
        if kind == "norm":
            return {"bytes": 2 * one + 2 * weights, "flops": 8 * case["rows"] * case["width"]}
        return {"bytes": 5 * one + 5 * weights, "flops": 24 * case["rows"] * case["width"]}
    if kind in ("adapted", "adapted_grad"):
        m, k, n, r = case["rows"], case["width"], case["n_out"], case["rank"]
        held = min(case["adapters"], m) * r * (k + n)
        if kind == "adapted":
            return {"bytes": 2 * (m * k + n * k + m * n + held) + 4 * m, "flops": 2 * m * (n * k + r * (n + k))}
        return {"bytes": 2 * (2 * m * k + 2 * n * k + 2 * m * n + 3 * held) + 4 * m, "flops": 2 * m * (2 * n * k + 4 * r * (n + k))}
    n, p = sum(_sizes(case)), DTYPES[case["param"]].itemsize
    each = 2 * p + DTYPES[case["grad"]].itemsize
    # 8 bits: codes read and written, two scales of every 256, and what the states stand for written
    return {"bytes": n * (each + 16) if case["bits"] == 32 else n * (each + 4 + 8) + n // BLOCK * 16, "flops": 20 * n}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _exact_adamw(case, s):
    (b1, b2), t, lr = HYPER["betas"], s["step"] + 1, HYPER["lr"]
    packed = lambda x: x.reshape(-1).double()[s["at"]]             # noqa: E731
    m, v = packed(s["m"]), packed(s["v"])
    if case["bits"] == 8:
        block = s["at"] // BLOCK
        m = torch.sign(m) * (m / 127) ** 2 * s["m_scale"].double()[block]
        v = (v / 255) ** 4 * s["v_scale"].double()[block]
    g = s["g"].double()
    m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g ** 2 - v)
    corrected = v.div(-math.expm1(t * math.log(b2)))
    p = s["p"].double()
    p = p - lr * HYPER["weight_decay"] * p - lr * m.div(-math.expm1(t * math.log(b1))) / (corrected ** 0.5 + HYPER["eps"])
    if case["bits"] == 8:
        def brought(x, most_code, power):
            a = torch.zeros(s["m_scale"].numel(), dtype=torch.float64, device=DEVICE).scatter_reduce_(0, block, x.abs(), "amax")
            a = a.float().double()[block]
            part = torch.where(a > 0, x.abs() / a, 0.0)
            code = torch.floor(most_code * part ** (1 / power) + 0.5).clamp(max=most_code)
            return a, torch.where((code == 0) & (x != 0) & (power == 4) & (a > 0), 1.0, code)

        a, code = brought(m, 127, 2)
        m = m.sign() * a * (code / 127) ** 2
        a, code = brought(v, 255, 4)
        v = a * (code / 255) ** 4
    whole = lambda x: torch.zeros(s["m"].numel(), dtype=torch.float64, device=DEVICE).index_put_((s["at"],), x)      # noqa: E731
    return {"p": p, "m": whole(m), "v": whole(v)}


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "adamw":
        return _exact_adamw(case, s)
    if kind in ("norm", "norm_grad"):
        grads = kind == "norm_grad"
        x, w, b = (s[t].double().requires_grad_(grads) for t in ("x", "weight", "bias"))
        each = x.view(case["groups"], -1, case["width"])
        var, mean = torch.var_mean(each, -1, correction=0, keepdim=True)
        y = ((each - mean) / (var + EPS).sqrt() * w.view(case["groups"], 1, -1) + b.view(case["groups"], 1, -1)).view_as(x)
        if not grads:
            return y
        dx, dw, db = torch.autograd.grad(y, (x, w, b), s["dy"].double())
        return {"y": y.detach(), "dx": dx, "dweight": dw, "dbias": db}
    grads = kind == "adapted_grad"
    x, down, up = (s[t].double().requires_grad_(grads) for t in ("x", "down", "up"))
    w = s["w"].double()
    parts = torch.zeros(case["rows"], case["n_out"], dtype=torch.float64, device=DEVICE)
    for g in range(case["adapters"]):
        rows = torch.nonzero(s["index"] == g)[:, 0]
        low = x.index_select(0, rows).mm(down[g].t()) * s["scales"][g].double()
        parts = parts.index_add(0, rows, low.mm(up[g].t()))
    y = x.mm(w.t()) + parts
    if not grads:
        return y
    dx, d_down, d_up = torch.autograd.grad(y, (x, down, up), s["dy"].double())
    return {"y": y.detach(), "dx": dx, "d_down": d_down, "d_up": d_up}
