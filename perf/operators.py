"""Performance cases of the operators around the cascaded attention of a layer.

A case is one pass through one of them, as a program built on the library makes it:

  norm       queries and keys of a packed projection: each head's RMS norm and the 3-axis rotation, in one pass
  norm_grad  the same in training: forward, then the gradients of queries, keys and both weights
  publish    the same in serving: K normed, rotated and published with V to the paged pool, Q normed and rotated
  i8         a linear map in 8-bit integers: the tokens' activations brought to 8 bits with a scale each, multiplied with
             weights held in 8 bits with a scale for each output channel
  gated      both projections of a gated feed-forward block, the activation and the product: act(x Wg') * (x Wu')
  gated_grad the same in training: forward, then the gradients of x and both weights

Sizes are the Wan shapes of `workloads` (12 heads and width 1536, 40 heads and width 5120, blocks of 3 x 30 x 52 tokens) with
feed-forward widths of 8/3 of the layer's, those of the tests, and single tokens.

The definitions.  Norm and rotation of a head's vector x of D values with weight w: y = w x / sqrt(mean(x^2) + eps), then pair j of
an axis with Da dims turns by position * theta^(-2j/Da).  8 bits: a row's scale is its largest magnitude over 127, its codes are
round-half-even(127 x / largest), an empty (all zero) row has scale 0 and codes 0; y = (codes . codes') * scale * scale'.
Activations: silu(g) = g / (1 + exp(-g)), gelu(g) = g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
FRAMES, THETA, EPS = 3, 10000.0, 1e-6
ROPE_DIMS = {32: (12, 10, 10), 64: (24, 20, 20), 128: (44, 42, 42)}
PAGE, WINDOW, MAX_INFLIGHT = 128, 6, 5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(kind, tokens, heads, grid_h, grid_w, first_frame, head_dim=128, dtype="bf16"):
    return {"kind": kind, "tokens": tokens, "heads": heads, "head_dim": head_dim, "grid_h": grid_h, "grid_w": grid_w,
            "first_frame": first_frame, "dtype": dtype}


def _publish(heads, grid_h, grid_w, blocks, first_block):
    return {"kind": "publish", "heads": heads, "grid_h": grid_h, "grid_w": grid_w, "blocks": blocks, "first_block": first_block}


def _i8(rows, n_out, k_in):
    return {"kind": "i8", "rows": rows, "n_out": n_out, "k_in": k_in}


def _gated(kind, rows, width, hidden, activation="silu"):
    return {"kind": kind, "rows": rows, "width": width, "hidden": hidden, "activation": activation}


def listed():
    return [
        # one token's queries and keys, 1.3B heads: all latency
        dict(_norm("norm", 1, 12, 30, 52, 18), name="norm_token"),
        # five blocks in flight at the 14B width: memory traffic
        dict(_norm("norm", 23400, 40, 30, 52, 18), name="norm_wan14b"),
        # gradients in fp32 at the tiny configuration's width, an odd number of tokens: a check beside a new model
        dict(_norm("norm_grad", 433, 2, 6, 8, 6, head_dim=64, dtype="f32"), name="norm_grad_f32"),
        # a training step on one block of the 1.3B model
        dict(_norm("norm_grad", 4680, 12, 30, 52, 0), name="norm_grad_wan1p3b"),
        # the smoke run's cascade published: small and ragged
        dict(_publish(3, 10, 13, 3, 2), name="publish_small"),
        # five blocks of the 14B model published: every layer and step of a rollout
        dict(_publish(40, 30, 52, 5, 6), name="publish_wan14b"),
        # one token through the 14B QKV projection: the weights' way from memory
        dict(_i8(1, 15360, 5120), name="i8_token"),
        # a few hundred tokens, odd sizes
        dict(_i8(257, 776, 1000), name="i8_odd"),
        # the 14B QKV projection of five blocks
        dict(_i8(23400, 15360, 5120), name="i8_wan14b_qkv"),
        # one token through the 14B feed-forward block's first half
        dict(_gated("gated", 1, 5120, 13824), name="gated_token"),
        # five blocks through it
        dict(_gated("gated", 23400, 5120, 13824), name="gated_wan14b"),
        # a training step on one block of the 1.3B model
        dict(_gated("gated_grad", 4680, 1536, 4096), name="gated_grad_wan1p3b"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _columns(rng, most):
    """A layer's usual widths, or odd multiples of 8"""
    if rng.random() < 0.5:
        return 128 * rng.choice([m for m in (1, 2, 3, 4, 6, 8, 9, 12, 15, 20, 32, 36, 40, 60, 70, 108, 120) if 128 * m <= most])
    return 8 * (2 * _log_int(rng, 8, most // 16) - 1)


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "publish", "i8", "i8", "gated", "gated", "gated_grad", "gated_grad"])
    rows = _log_int(rng, 1, 23400)
    if kind in ("norm", "norm_grad"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return _norm(kind, rows, rng.choice([1, 2, 3, 5, 8, 12, 16, 40]), _log_int(rng, 1, 30), _log_int(rng, 1, 52),
                     rng.randint(0, 60), 128 if dtype == "bf16" else rng.choice([32, 64, 128]), dtype)
    if kind == "publish":
        blocks = rng.randint(1, MAX_INFLIGHT)
        return _publish(rng.choice([1, 2, 3, 6, 8, 12, 16, 40]), _log_int(rng, 2, 30), _log_int(rng, 3, 52), blocks,
                        rng.randint(0, WINDOW + MAX_INFLIGHT - blocks))
    if kind == "i8":
        return _i8(rows, _columns(rng, 15360), _log_int(rng, 64, 5120))
    width = 128 * rng.choice([1, 2, 3, 5, 8, 12, 16, 20, 30, 40])
    if kind == "gated_grad":
        rows = max(1, rows // 3)                                   # no more work than the largest listed case
    return _gated(kind, rows, width, _columns(rng, 13824), rng.choice(["silu", "gelu"]))


# ------------------------------------------------------------------------------------------------ inputs

def _inputs(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dtype)

    kind = case["kind"]
    if kind == "i8":
        m, n, k = case["rows"], case["n_out"], case["k_in"]
        x = normal(m, k, dtype=torch.float32)
        x *= torch.exp(0.5 * normal(k, dtype=torch.float32))      # channels differ in size, as a layer's activations do
        return {"x": x.to(torch.bfloat16), "w": normal(n, k, scale=k ** -0.5)}
    if kind in ("gated", "gated_grad"):
        m, k, f = case["rows"], case["width"], case["hidden"]
        s = {"x": normal(m, k), "w_gate": normal(f, k, scale=k ** -0.5), "w_up": normal(f, k, scale=k ** -0.5)}
        if kind == "gated_grad":
            s["dh"] = normal(m, f)
        return s
    H = case["heads"]
    if kind == "publish":
        L, D, dtype = FRAMES * case["grid_h"] * case["grid_w"], 128, torch.bfloat16
        n = case["blocks"] * L
    else:
        n, D, dtype = case["tokens"], case["head_dim"], DTYPES[case["dtype"]]
    qkv = normal(n, 3, H, D, dtype=dtype)                          # as the projection leaves it
    s = {"q": qkv[:, 0], "k": qkv[:, 1], "v": qkv[:, 2]}
    for name in ("q_weight", "k_weight"):
        s[name] = (1 + 0.2 * normal(D, dtype=torch.float32)).to(dtype)
    if kind == "norm_grad":
        s["dq_out"], s["dk_out"] = normal(n, H, D, dtype=dtype), normal(n, H, D, dtype=dtype)
    return s


def _pool(case):
    from paper_2511_20426_amd.runner import CascadePool
    D, dtype = case.get("head_dim", 128), case.get("dtype", "bf16")
    return CascadePool(heads=case["heads"], head_dim=D, frames_per_block=FRAMES, grid_h=case["grid_h"], grid_w=case["grid_w"],
                       rope_dims=ROPE_DIMS[D], rope_theta=THETA, sink_blocks=0,
                       window_blocks=WINDOW if case["kind"] == "publish" else 0,
                       max_inflight=MAX_INFLIGHT if case["kind"] == "publish" else 1, page_tokens=PAGE, dtype=dtype, device=DEVICE)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "i8":                                               # the weights are held in 8 bits
        codes, scales = _codes(s.pop("w"))
        s["w_codes"], s["w_scales"] = codes.to(torch.int8), scales
        if own:
            from paper_2511_20426_amd.runner import QuantizedRows
            s["w"] = QuantizedRows.from_codes(s["w_codes"], s["w_scales"])
            s["y"] = torch.empty((case["rows"], case["n_out"]), dtype=torch.bfloat16, device=DEVICE)
    elif kind == "gated" and own:
        s["h"] = torch.empty((case["rows"], case["hidden"]), dtype=torch.bfloat16, device=DEVICE)
    elif kind not in ("gated", "gated_grad") and own:
        pool = s["pool"] = _pool(case)
        s["q_out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEVICE)
        if kind == "publish":
            L, C, H = pool.block_tokens, case["blocks"], case["heads"]
            s["ids"], s["timesteps"] = list(range(case["first_block"], case["first_block"] + C)), [0, 250, 500, 750, 1000][:C]
            s["ks"], s["vs"] = ([s[t][i * L:(i + 1) * L] for i in range(C)] for t in "kv")
            pages = -(-L // PAGE)
            # the pages of the blocks in flight: consecutive slots of the pool
            each = pages * H * 2 * PAGE * 128 * 2
            s["pages"] = pool.pool[case["first_block"] * each:(case["first_block"] + C) * each].view(torch.bfloat16).view(
                C, pages, H, 2, PAGE, 128)
        else:
            s["k_out"] = torch.empty(s["k"].shape, dtype=s["k"].dtype, device=DEVICE)
    return s


# ------------------------------------------------------------------------------------------------ the plain forms

def _angles(case, first_frame, n):
    """cos and sin [n, D / 2] of the tokens' rotation; angles in 64 bits."""
    D, gh, gw = case.get("head_dim", 128), case["grid_h"], case["grid_w"]
    t = torch.arange(n, device=DEVICE)
    axes = (first_frame + t // (gh * gw), t // gw % gh, t % gw)
    parts = []
    for pos, dims in zip(axes, ROPE_DIMS[D]):
        freq = THETA ** (-2.0 * torch.arange(dims // 2, device=DEVICE, dtype=torch.float64) / dims)
        parts.append(pos[:, None].double() * freq)
    angle = torch.cat(parts, 1)
    return angle.cos().float(), angle.sin().float()


def _norm_rope(x, w, cos, sin):
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    u, v = y[..., 0::2], y[..., 1::2]
    c, s = cos[:, None], sin[:, None]
    return torch.stack((u * c - v * s, u * s + v * c), -1).flatten(-2)


def _norm_rope_grad(dz, x, w, cos, sin):
    x, w, dz = x.float(), w.float(), dz.float()
    a, b = dz[..., 0::2], dz[..., 1::2]
    c, s = cos[:, None], sin[:, None]
    dy = torch.stack((a * c + b * s, b * c - a * s), -1).flatten(-2)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    normed = x * r
    dw = (dy * normed).sum((0, 1), dtype=torch.float64).float()
    dn = dy * w
    return r * (dn - normed * (dn * normed).mean(-1, keepdim=True)), dw


def _pages(k, v):
    """The pool's pages of one block [pages, heads, 2, 128, 128] from its K and V [tokens, heads, 128]: K's rows are tokens, V's
    dims, with tokens in an order of their own; the sixteen chunks of 8 values of row r lie at chunk ^ (r % 16); zeros behind
    the block's end."""
    L, H, D = k.shape
    pages = -(-L // PAGE)

    def whole(t):
        return torch.cat((t, t.new_zeros(pages * PAGE - L, H, D))).view(pages, PAGE, H, D)

    row, chunk = torch.arange(128, device=DEVICE)[:, None], torch.arange(16, device=DEVICE)[None]
    stored = ((chunk ^ (row % 16))[:, :, None] * 8 + torch.arange(8, device=DEVICE)).flatten(1)           # [128, 128]
    perm = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device=DEVICE)
    order = (torch.arange(0, 128, 16, device=DEVICE)[:, None] + perm).flatten()
    kp = whole(k).permute(0, 2, 1, 3)
    vp = whole(v).permute(0, 2, 3, 1)[..., order]
    return torch.stack([t.gather(3, stored.expand(pages, H, 128, 128)) for t in (kp, vp)], 2)


def _codes(x):
    """Codes (whole numbers in 32-bit floats) and scales of x's rows; the quotient in 64 bits, for values next to a border."""
    x = x.double()
    most = x.abs().amax(1, keepdim=True)
    codes = torch.where(most > 0, torch.round(x * 127 / most), torch.zeros_like(x))
    return codes.float(), most[:, 0].float() / 127


def _act(g, activation):
    if activation == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g)))


def _act_grad(g, activation):
    if activation == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "i8":
        codes, scales = _codes(s["x"])
        return ((codes @ s["w_codes"].float().T) * scales[:, None] * s["w_scales"]).to(torch.bfloat16)
    if kind in ("gated", "gated_grad"):
        act = case["activation"]
        x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
        g, u = x @ wg.T, x @ wu.T
        a = _act(g, act)
        h = (a * u).to(torch.bfloat16)
        if kind == "gated":
            return h
        dh = s["dh"].float()
        dg, du = dh * u * _act_grad(g, act), dh * a
        grads = {"dx": dg @ wg + du @ wu, "dw_gate": dg.T @ x, "dw_up": du.T @ x}
        return {"h": h, **{name: t.to(torch.bfloat16) for name, t in grads.items()}}
    dtype = s["q"].dtype
    if kind == "publish":
        L, first = FRAMES * case["grid_h"] * case["grid_w"], FRAMES * case["first_block"]
    else:
        first = case["first_frame"]
    cos, sin = _angles(case, first, s["q"].shape[0])
    q = _norm_rope(s["q"], s["q_weight"], cos, sin).to(dtype)
    k = _norm_rope(s["k"], s["k_weight"], cos, sin).to(dtype)
    if kind == "norm":
        return {"q": q, "k": k}
    if kind == "publish":
        return {"q": q, "pages": torch.stack([_pages(k[i:i + L], s["v"][i:i + L]) for i in range(0, k.shape[0], L)])}
    dq, dqw = _norm_rope_grad(s["dq_out"], s["q"], s["q_weight"], cos, sin)
    dk, dkw = _norm_rope_grad(s["dk_out"], s["k"], s["k_weight"], cos, sin)
    return {"q": q, "k": k, "dq": dq.to(dtype), "dk": dk.to(dtype), "dq_weight": dqw, "dk_weight": dkw}


# ------------------------------------------------------------------------------------------------ the operators

def run(s):
    if not own:
        return _plain(s)
    from paper_2511_20426_amd import runner
    case = s["case"]
    kind = case["kind"]
    if kind == "i8":
        return runner.linear_i8(s["x"], s["w"], out=s["y"])
    if kind == "gated":
        return runner.gated_linear(s["x"], s["w_gate"], s["w_up"], case["activation"], out=s["h"])
    if kind == "gated_grad":
        h, saved = runner.gated_linear_train(s["x"], s["w_gate"], s["w_up"], case["activation"])
        dx, dw_gate, dw_up = runner.gated_linear_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], saved, case["activation"])
        return {"h": h, "dx": dx, "dw_gate": dw_gate, "dw_up": dw_up}
    pool, weights = s["pool"], (s["q_weight"], s["k_weight"])
    if kind == "publish":
        pool.append_batch(s["ids"], s["timesteps"], 0, s["ks"], s["vs"], k_weight=s["k_weight"], eps=EPS)
        q, _ = pool.qk_norm_rope(s["q"], None, s["q_weight"], None, FRAMES * case["first_block"], eps=EPS, q_out=s["q_out"])
        return {"q": q, "pages": s["pages"]}
    q, k = pool.qk_norm_rope(s["q"], s["k"], *weights, case["first_frame"], eps=EPS, q_out=s["q_out"], k_out=s["k_out"])
    if kind == "norm":
        return {"q": q, "k": k}
    dq, dk, dqw, dkw = pool.qk_norm_rope_backward(s["dq_out"], s["dk_out"], s["q"], s["k"], *weights, case["first_frame"], eps=EPS)
    return {"q": q, "k": k, "dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}


def work(case):
    kind = case["kind"]
    if kind == "i8":
        m, n, k = case["rows"], case["n_out"], case["k_in"]
        return {"bytes": 2 * m * k + n * k + 4 * n + 2 * m * n, "flops": 2 * m * n * k}
    if kind in ("gated", "gated_grad"):
        m, k, f = case["rows"], case["width"], case["hidden"]
        one = 2 * (m * k + 2 * f * k + m * f)
        return {"bytes": one, "flops": 4 * m * f * k} if kind == "gated" else {"bytes": 2 * one, "flops": 12 * m * f * k}
    if kind == "publish":
        one = case["blocks"] * FRAMES * case["grid_h"] * case["grid_w"] * case["heads"] * 128
        return {"bytes": 6 * 2 * one, "flops": 2 * 7 * one}
    one = case["tokens"] * case["heads"] * case["head_dim"]
    size = 2 if case["dtype"] == "bf16" else 4
    return {"bytes": 4 * size * one, "flops": 2 * 7 * one} if kind == "norm" else {"bytes": 8 * size * one, "flops": 2 * 25 * one}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _turned(case, first_frame, x, w):
    """Norm and rotation as products of complex numbers."""
    D, plane = case.get("head_dim", 128), case["grid_h"] * case["grid_w"]
    n = x.shape[0]
    turn = torch.empty(n, D // 2, dtype=torch.complex128, device=DEVICE)
    pair = 0
    for axis, dims in enumerate(ROPE_DIMS[D]):
        for j in range(dims // 2):
            token = torch.arange(n, device=DEVICE, dtype=torch.int64)
            pos = (first_frame + token.div(plane, rounding_mode="floor"), token.remainder(plane).div(case["grid_w"], rounding_mode="floor"),
                   token.remainder(case["grid_w"]))[axis]
            angle = pos.double() / THETA ** (2.0 * j / dims)
            turn[:, pair] = torch.polar(torch.ones_like(angle), angle)
            pair += 1
    y = w.double() * x / (x.square().sum(-1, keepdim=True) / D + EPS).sqrt()
    z = torch.view_as_complex(y.unflatten(-1, (D // 2, 2))) * turn[:, None]
    return torch.view_as_real(z).flatten(-2)


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "i8":
        def whole(t):
            most = t.double().abs().max(1).values
            return torch.round(t.double() * 127 / torch.where(most > 0, most, 1.0)[:, None]), most / 127

        (cx, sx), (cw, sw) = whole(s["x"]), whole(s["w"])
        return torch.outer(sx, sw) * cx.mm(cw.t())
    if kind in ("gated", "gated_grad"):
        grads = kind == "gated_grad"
        x, wg, wu = (s[t].double().requires_grad_(grads) for t in ("x", "w_gate", "w_up"))
        g = x.mm(wg.t())
        h = (g * torch.sigmoid(g) if case["activation"] == "silu" else torch.nn.functional.gelu(g, approximate="tanh")) * x.mm(wu.t())
        if not grads:
            return h
        dx, dwg, dwu = torch.autograd.grad(h, (x, wg, wu), s["dh"].double())
        return {"h": h.detach(), "dx": dx, "dw_gate": dwg, "dw_up": dwu}
    if kind == "publish":
        first = FRAMES * case["first_block"]
        L, C, H = FRAMES * case["grid_h"] * case["grid_w"], case["blocks"], case["heads"]
        q = _turned(case, first, s["q"].double(), s["q_weight"])
        k = _turned(case, first, s["k"].double(), s["k_weight"])
        count = -(-L // PAGE)
        rows = torch.zeros(2, C, count * PAGE, H, 128, dtype=torch.float64, device=DEVICE)
        rows[0, :, :L], rows[1, :, :L] = k.view(C, L, H, 128), s["v"].double().reshape(C, L, H, 128)
        rows = rows.view(2, C, count, PAGE, H, 128)
        pages = torch.empty(C, count, H, 2, PAGE, 128, dtype=torch.float64, device=DEVICE)
        place = torch.arange(128, device=DEVICE)
        for r in range(128):                                       # what lies in row r of a page
            held = (place // 8 ^ r % 16) * 8 + place % 8           # of K the dim, of V the token's number in its order
            token = 16 * (held // 16) + 4 * (held // 8 % 2) + held % 4 + 8 * (held % 8 // 4)
            pages[:, :, :, 0, r] = rows[0, :, :, r][..., held]
            pages[:, :, :, 1, r] = rows[1, :, :, :, :, r][:, :, token].transpose(2, 3)
        return {"q": q, "pages": pages}
    first = case["first_frame"]
    grads = kind == "norm_grad"
    q, k, wq, wk = (s[t].double().requires_grad_(grads) for t in ("q", "k", "q_weight", "k_weight"))
    q_out, k_out = _turned(case, first, q, wq), _turned(case, first, k, wk)
    if not grads:
        return {"q": q_out, "k": k_out}
    dq, dk, dqw, dkw = torch.autograd.grad((q_out, k_out), (q, k, wq, wk), (s["dq_out"].double(), s["dk_out"].double()))
    return {"q": q_out.detach(), "k": k_out.detach(), "dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
