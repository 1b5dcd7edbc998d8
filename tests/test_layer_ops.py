"""The operators around the attention of a layer (norms of queries and keys with the rotation, 8-bit linear maps, gated projections)
against plain implementations in 64 bits, their gradients against the formulas' and against differences, and their refusals."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2511_20426_amd import binding as B

ROPE = {32: (12, 10, 10), 64: (24, 20, 20), 128: (44, 42, 42)}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}        # a rounding, relative: half a step
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _normal(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(dtype).to(DEV)


def _pool(heads, D=128, grid=(4, 5), dtype="bf16", frames=3, inflight=2):
    from paper_2511_20426_amd.runner import CascadePool
    return CascadePool(heads=heads, head_dim=D, frames_per_block=frames, grid_h=grid[0], grid_w=grid[1], rope_dims=ROPE[D], rope_theta=10000.0,
                       sink_blocks=0, window_blocks=2, max_inflight=inflight, page_tokens=128, dtype=dtype)


# ------------------------------------------------------------------------------------------------ plain implementations, 64 bits

def _angles(D, grid, first, n):
    t = torch.arange(n, dtype=torch.float64)
    plane = grid[0] * grid[1]
    axes = (first + torch.floor(t / plane), torch.floor(t % plane / grid[1]), t % plane % grid[1])
    return torch.cat([p[:, None] * 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d) for p, d in zip(axes, ROPE[D])], 1)


def _rotate(y, ang):
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    u, v = y[..., 0::2], y[..., 1::2]
    return torch.stack((u * c - v * s, u * s + v * c), -1).flatten(-2)


def _norm_rope(x, w, eps, ang):
    return _rotate(w * x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps), ang)


def _pairs(t):
    """of each value the sum of magnitudes of its pair: what the errors of a rotation's fp32 products go by"""
    return (t[..., 0::2].abs() + t[..., 1::2].abs()).repeat_interleave(2, -1)


def _act(g, name):
    return g * torch.sigmoid(g) if name == "silu" else torch.nn.functional.gelu(g, approximate="tanh")


# ------------------------------------------------------------------------------------------------ norms and rotation

# fp32 on the way: a sum of up to 128 squares (8 in a chain, 4 exchanges, under a root), 3 products, the rotation's 2 and its cos / sin (1e-7
# each on the reduced angle for bf16, correctly rounded for fp32): less than 16 roundings of 2^-24
WAY = 16 * 2.0 ** -24

NORMS = [("bf16", 128, 3, 1, (4, 5), 0), ("bf16", 128, 1, 5, (1, 1), 7), ("bf16", 128, 5, 67, (3, 7), 2), ("bf16", 128, 40, 9, (30, 52), 18),
         ("bf16", 128, 2, 300, (5, 3), 5000), ("f32", 128, 2, 33, (2, 3), 1), ("f32", 64, 3, 131, (6, 8), 4), ("f32", 32, 1, 1, (2, 2), 0),
         ("f32", 32, 9, 66, (1, 4), 90000)]


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["both", "q", "k"])
@pytest.mark.parametrize("dtype,D,heads,n,grid,first", NORMS)
def test_norm_rope(dtype, D, heads, n, grid, first, which):
    """Strided views of a packed projection; a head of zeros, one of a single large value, values of 1e-18 (their squares are below fp32's eps
    beside 1e-6)."""
    pool, gen, t = _pool(heads, D, grid, dtype), _gen(n + D), {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    qkv = _normal(gen, n, 3, heads, D, dtype=t)
    qkv[0, 0, 0] = 0
    qkv[0, 1, 0] = 0
    qkv[0, 1, 0, D // 2] = 1000
    qkv[n - 1, 0, heads - 1] *= 1e-18
    weights = [_normal(gen, D, dtype=t) for _ in range(2)]
    sides = {"both": (0, 1), "q": (0,), "k": (1,)}[which]
    args = [(qkv[:, s], weights[s]) if s in sides else (None, None) for s in range(2)]
    keep = qkv.clone()
    outs = pool.qk_norm_rope(args[0][0], args[1][0], args[0][1], args[1][1], first)
    assert (qkv == keep).all()
    ang = _angles(D, grid, first, n)
    for s in range(2):
        if s not in sides:
            assert outs[s] is None
            continue
        x, w = qkv[:, s].double().cpu(), weights[s].double().cpu()
        ref = _norm_rope(x, w, 1e-6, ang)
        bound = ref.abs() * HALF[t] + _pairs(ref) * 2 * WAY + 1e-30
        assert ((outs[s].double().cpu() - ref).abs() <= bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_norm_rope_in_place_into_strides_and_on_a_stream(dtype, D):
    pool, gen, t = _pool(3, D, (4, 5), dtype), _gen(3), {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    qkv, w = _normal(gen, 50, 3, 3, D, dtype=t), _normal(gen, D, dtype=t)
    q, k = pool.qk_norm_rope(qkv[:, 0], qkv[:, 1], w, w, 4)
    wide = torch.full((50, 4, 3, D + 8), 7.0, dtype=t, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        pool.qk_norm_rope(qkv[:, 0], qkv[:, 1], w, w, 4, q_out=wide[:, 1, :, :D], k_out=qkv[:, 1])
    torch.cuda.current_stream().wait_stream(s)
    assert (wide[:, 1, :, :D] == q).all() and (qkv[:, 1] == k).all()
    assert (wide[:, 0] == 7).all() and (wide[:, 2:] == 7).all() and (wide[:, 1, :, D:] == 7).all()


def _norm_grads(dz, x, w, eps, ang):
    """dx, dw and the magnitudes that their fp32 errors go by"""
    D = x.shape[-1]
    dy = _rotate(dz, -ang)
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n, dn = x * r, dy * w
    dx = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    size = _pairs(dy) * w.abs()
    return dx, (dy * n).sum((0, 1)), r * (size + n.abs() * (size * n.abs()).sum(-1, keepdim=True) / D), (_pairs(dy) * n.abs()).sum((0, 1))


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["both", "q", "k"])
@pytest.mark.parametrize("dtype,D,heads,n,grid,first", NORMS + [("bf16", 128, 12, 2345, (30, 52), 0), ("bf16", 128, 1, 4100, (3, 3), 0)])
def test_norm_rope_backward(dtype, D, heads, n, grid, first, which):
    pool, gen, t = _pool(heads, D, grid, dtype), _gen(n + D + 1), {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    qkv, dz = _normal(gen, n, 3, heads, D, dtype=t), _normal(gen, n, heads, 2, D, dtype=t)
    qkv[0, 0, 0] = 0                              # (its gradient is dn / sqrt(eps))
    weights = [_normal(gen, D, dtype=t) for _ in range(2)]
    sides = {"both": (0, 1), "q": (0,), "k": (1,)}[which]
    pick = lambda f: [f(s) if s in sides else None for s in range(2)]  # noqa: E731
    call = lambda: pool.qk_norm_rope_backward(*pick(lambda s: dz[:, :, s]), *pick(lambda s: qkv[:, s]), *pick(lambda s: weights[s]), first)  # noqa: E731
    got, again = call(), call()
    ang = _angles(D, grid, first, n)
    for s in range(2):
        if s not in sides:
            assert got[s] is None and got[2 + s] is None
            continue
        x, w, d = (v.double().cpu() for v in (qkv[:, s], weights[s], dz[:, :, s]))
        dx, dw, size, size_w = _norm_grads(d, x, w, 1e-6, ang)
        assert ((got[s].double().cpu() - dx).abs() <= dx.abs() * HALF[t] + size * 3 * WAY + 1e-30).all()
        # a lane sums in fp32 over the tokens and heads that it meets: at most n heads / 4 in a chain, 64 at these sizes and more at once
        assert ((got[2 + s].double().cpu() - dw).abs() <= size_w * (2 * WAY + 128 * 2.0 ** -24) + 1e-30).all()
        assert (got[s] == again[s]).all() and (got[2 + s] == again[2 + s]).all()      # the same bits every time
        # ... and the formula against differences of the forward
        step, move, move_w = 1e-5, torch.randn(x.shape, generator=gen, dtype=torch.float64), torch.randn(w.shape, generator=gen, dtype=torch.float64)
        x1, part = x[-1:], ang[-1:]               # (the last token: a head of zeros bends too much for a step)
        along = sum(sg * (d[-1:] * _norm_rope(x1 + sg * step * move[-1:], w, 1e-6, part)).sum() for sg in (1, -1)) / (2 * step)
        if not (n == 1 and s == 0):
            assert abs(along - (dx[-1:] * move[-1:]).sum()) <= 1e-5 * (dx[-1:].abs() * move[-1:].abs()).sum() + 1e-6
        along = sum(sg * (d * _norm_rope(x, w + sg * step * move_w, 1e-6, ang)).sum() for sg in (1, -1)) / (2 * step)
        assert abs(along - (dw * move_w).sum()) <= 1e-6 * (size_w * move_w.abs()).sum()


@pytest.mark.gpu
def test_norm_rope_of_no_tokens():
    pool = _pool(2)
    q, w = torch.empty((0, 2, 128), dtype=torch.bfloat16, device=DEV), torch.ones(128, dtype=torch.bfloat16, device=DEV)
    assert pool.qk_norm_rope(q, q, w, w, 0)[0].shape == (0, 2, 128)
    dq, dk, dqw, dkw = pool.qk_norm_rope_backward(q, q, q, q, w, w, 0)
    assert dq.shape == dk.shape == (0, 2, 128) and (dqw == 0).all() and (dkw == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D,heads,grid,blocks", [("bf16", 128, 2, (5, 7), [3, 4]), ("bf16", 128, 1, (1, 2), [0]), ("bf16", 128, 40, (6, 11), [2, 3]),
                                                       ("bf16", 128, 12, (20, 20), [1, 2]), ("f32", 64, 2, (5, 9), [5]), ("f32", 32, 3, (2, 2), [0, 1])])
def test_normed_keys_in_the_pool(dtype, D, heads, grid, blocks):
    """Published on the way, K has the bits of qk_norm_rope's keys at every page, V those of an append without norm."""
    gen, t = _gen(heads), {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    L = 3 * grid[0] * grid[1]
    qkv, w = _normal(gen, len(blocks) * L, 3, heads, D, dtype=t), _normal(gen, D, dtype=t)
    ks, vs = [qkv[i * L:(i + 1) * L, 1] for i in range(len(blocks))], [qkv[i * L:(i + 1) * L, 2] for i in range(len(blocks))]
    a, b = _pool(heads, D, grid, dtype), _pool(heads, D, grid, dtype)
    assert a.append_batch(blocks, [0] * len(blocks), 0, ks, vs, k_weight=w, eps=1e-5) == b.append_batch(blocks, [0] * len(blocks), 0, ks, vs)
    normed = a.qk_norm_rope(None, qkv[:, 1], None, w, 3 * blocks[0], eps=1e-5)[1]
    # the pool's rotation is undone by no one: pages of normed K are compared through an append of K that is rotated back in fp64
    pages = -(-L // 128)
    per = 2 * 128 * D
    for i, g in enumerate(blocks):
        for p in range(pages):
            for h in range(heads):
                at = a.ctx.kv_cache_page_index(g, p, h)
                ka, kb = (x.pool[at * per * t.itemsize:(at + 1) * per * t.itemsize].view(t).view(2, 128, D) for x in (a, b))
                assert (ka[1] == kb[1]).all()
                k = ka[0]
                if dtype == "bf16":
                    c = torch.arange(16, device=DEV)[None] ^ (torch.arange(128, device=DEV)[:, None] & 15)
                    k = k.view(128, 16, 8).gather(1, c[:, :, None].expand(128, 16, 8)).view(128, D)
                rows = min(128, L - 128 * p)
                assert (k[:rows] == normed[i * L + 128 * p:i * L + 128 * p + rows, h]).all() and (k[rows:] == 0).all()


@pytest.mark.gpu
def test_attention_over_normed_keys():
    """A small cascade: published normed keys and normed queries against softmax attention in 64 bits."""
    gen, grid, heads = _gen(11), (4, 6), 2
    pool, L = _pool(heads, 128, grid), 72
    qkv, wq, wk = _normal(gen, 2 * L, 3, heads, 128), _normal(gen, 128), _normal(gen, 128)
    pool.append_batch([0, 1], [0, 0], 0, [qkv[:L, 1], qkv[L:, 1]], [qkv[:L, 2], qkv[L:, 2]], k_weight=wk)
    q, _ = pool.qk_norm_rope(qkv[:, 0], None, wq, None, 0)
    got = pool.forward(q, [0, 1], B.CA_BIDIRECTIONAL).double().cpu()
    ang = _angles(128, grid, 0, 2 * L)
    qr, kr = (_norm_rope(qkv[:, s].double().cpu(), w.double().cpu(), 1e-6, ang).transpose(0, 1) for s, w in ((0, wq), (1, wk)))
    ref = torch.softmax(qr @ kr.transpose(1, 2) / 128 ** 0.5, -1) @ qkv[:, 2].double().cpu().transpose(0, 1)
    # the bound of the attention tests: 5e-3 of the norm
    assert (got.transpose(0, 1) - ref).norm() <= 5e-3 * ref.norm()


# ------------------------------------------------------------------------------------------------ 8 bits

def _exact_codes(x):
    """round-half-even(127 x / largest) in whole numbers: doubles hold every 24-bit value as integer * 2^e exactly"""
    from fractions import Fraction
    out = np.zeros(x.shape, np.int64)
    for r in range(x.shape[0]):
        most = max(abs(Fraction(float(v))) for v in x[r])
        if most:
            out[r] = [round(127 * Fraction(float(v)) / most) for v in x[r]]      # (of a Fraction: half to even)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,k,pad,off", [(1, 1, 0, 0), (3, 7, 1, 0), (2, 100, 0, 0), (5, 257, 7, 3), (4, 2600, 8, 0), (1100, 24, 0, 0), (1025, 40, 9, 1)])
def test_quantize_rows(dtype, rows, k, pad, off):
    """Codes of exact arithmetic: random values, ties (values of (n + 1/2) / 127 of the largest), values beside them, rows that leave fp32's range
    times 127 or whose reciprocal does; rows that are not aligned."""
    from paper_2511_20426_amd.runner import quantize_rows
    gen = _gen(rows + k)
    x = torch.randn(rows, k, generator=gen, dtype=torch.float64)
    for r in range(rows):                         # (a largest value of 127 * 2^e: ties are representable)
        if r % 3 == 1:
            x[r, :] = (torch.randint(-127, 127, (k,), generator=gen) + 0.5) * 2.0 ** (r % 5)
            x[r, r % k] = 127 * 2.0 ** (r % 5)
        if r % 7 == 2:
            x[r] *= 2.0 ** 116
        if r % 7 == 3:
            x[r] *= 2.0 ** -128
    if rows > 4:
        x[4] = 0
    x = x.to(dtype)
    if dtype == torch.float32 and rows > 1:       # one step beside a tie, either way
        x[1] = torch.nextafter(x[1], torch.where(torch.rand(k, generator=gen) < 0.5, torch.inf, -torch.inf).float())
    whole = torch.zeros(rows * (k + pad) + off, dtype=dtype, device=DEV)
    view = whole[off:].view(rows, k + pad)[:, :k]
    view.copy_(x)
    got = quantize_rows(view)
    want = _exact_codes(x.double().numpy())
    codes = got.codes.cpu().numpy().astype(np.int64)
    assert codes.shape == (rows, -(-k // 256) * 256) and (codes[:, k:] == 0).all()
    assert (codes[:, :k] == want).all(), np.argwhere(codes[:, :k] != want)[:5]
    most = x.double().abs().amax(1)
    assert ((got.scales.double().cpu() - most / 127).abs() <= most / 127 * 2.0 ** -23 + 2.0 ** -149).all()


@pytest.mark.gpu
def test_rows_that_are_not_finite():
    """... have scale NaN and codes 0, their neighbours keep theirs; their outputs are NaN, the others' finite."""
    from paper_2511_20426_amd.runner import linear_i8, quantize_rows
    gen = _gen(5)
    for rows in (4, 6, 1030):
        x, w = _normal(gen, rows, 300), _normal(gen, 16, 300)
        x[1, 7], x[3, 299], x[rows - 1, 0] = float("inf"), float("nan"), -float("inf")
        bad = torch.zeros(rows, dtype=torch.bool, device=DEV)
        bad[[1, 3, rows - 1]] = True
        q = quantize_rows(x)
        assert (q.scales.isnan() == bad).all() and (q.codes[bad] == 0).all()
        fine = quantize_rows(torch.where(bad[:, None], torch.zeros_like(x), x))
        assert (q.codes[~bad] == fine.codes[~bad]).all() and (q.scales[~bad] == fine.scales[~bad]).all()
        y = linear_i8(x, quantize_rows(w))
        assert y[bad].isnan().all() and y[~bad].isfinite().all()


def _i8_bound(ref):
    # the sum is exact; made fp32, two products, one rounding to bf16
    return ref.abs() * (2.0 ** -8 + 4 * 2.0 ** -24) + 1e-38


I8 = [(1, 8, 1), (1, 8, 8), (1, 776, 1000), (2, 40, 6144), (4, 72, 6144), (3, 88, 6152), (5, 136, 640), (4, 24, 1001), (3, 24, 255), (16, 64, 256), (17, 40, 257), (32, 136, 5120), (33, 8, 300), (64, 128, 512), (65, 200, 90), (129, 72, 640),
      (300, 1032, 2000), (1100, 1400, 256), (2050, 1160, 128), (2050, 2184, 1000), (4680, 1544, 384), (700, 9000, 513)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", I8)
def test_linear_i8(M, N, K):
    """Against whole-number products; nothing outside the result is written."""
    from paper_2511_20426_amd.runner import QuantizedRows, linear_i8, quantize_rows
    gen = _gen(M + N + K)
    x, w = (torch.randint(-127, 128, (n, K), generator=gen, dtype=torch.int8).to(DEV) for n in (M, N))
    x[0] = 127                                    # (sums as large as they come)
    w[0] = -127
    xs, ws = (torch.rand(n, generator=gen).to(DEV) + 0.01 for n in (M, N))
    y = torch.full((M + 2, N + 16), 7.0, dtype=torch.bfloat16, device=DEV)
    linear_i8(QuantizedRows.from_codes(x, xs), QuantizedRows.from_codes(w, ws), out=y[:M, :N])
    torch.cuda.synchronize()
    assert (y[M:] == 7).all() and (y[:, N:] == 7).all()
    # (doubles hold the sums)
    ref = (x.double().cpu() @ w.double().cpu().T) * xs.double().cpu()[:, None] * ws.double().cpu()
    assert ((y[:M, :N].double().cpu() - ref).abs() <= _i8_bound(ref)).all()
    # from bf16 activations: codes by quantize_rows
    xb = _normal(gen, M, K)
    q, wq = quantize_rows(xb), QuantizedRows.from_codes(w, ws)
    ref = (q.codes[:, :K].double().cpu() @ w.double().cpu().T) * q.scales.double().cpu()[:, None] * ws.double().cpu()
    assert ((linear_i8(xb, wq).double().cpu() - ref).abs() <= _i8_bound(ref)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("off,pad", [(0, 0), (1, 3), (8, 8)])
@pytest.mark.parametrize("M,N,K", [(1, 40, 7), (1, 24, 8), (1, 512, 230), (2, 72, 9), (4, 40, 255), (5, 24, 257), (8, 8200, 65), (9, 8200, 65), (9, 136, 1001), (12, 40, 1536),
                                   (12, 264, 1535), (13, 40, 1536), (1, 40, 1537), (2, 136, 6143), (2, 24, 6144), (1, 40, 6145), (2, 12296, 1600), (3, 24, 2000)])
def test_few_tokens_of_any_alignment_in_8_bits(M, N, K, off, pad):
    """The calls that make the codes on their way give the bits of those that have them made ahead; NaN and rows of zeros stay in their rows."""
    from paper_2511_20426_amd.runner import linear_i8, quantize_rows
    gen = _gen(M + N + K + off)
    whole = _normal(gen, M * (K + pad) + off)
    x = whole[off:].view(M, K + pad)[:, :K]
    w = quantize_rows(_normal(gen, N, K))
    if M > 2:
        x[0] = 0
        x[2, K - 1] = float("nan")
    y = linear_i8(x, w)
    ahead = linear_i8(quantize_rows(x), w)
    bad = torch.zeros(M, dtype=torch.bool, device=DEV)
    bad[2:3] = M > 2
    assert (y[~bad] == ahead[~bad]).all() and y[bad].isnan().all() and ahead[bad].isnan().all()
    if M > 2:
        assert (y[0] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 40])
def test_linear_i8_at_the_longest_k(M):
    from paper_2511_20426_amd.runner import QuantizedRows, linear_i8
    K = B.CA_I8_MAX_K
    x, w = (torch.full((n, K), 127, dtype=torch.int8, device=DEV) for n in (M, 8))
    w[1] = -127
    one = torch.ones(max(M, 8), device=DEV)
    y = linear_i8(QuantizedRows(x, one[:M], K), QuantizedRows(w, one[:8].contiguous(), K)).double().cpu()
    ref = torch.full((M, 8), 127.0 * 127 * K, dtype=torch.float64)
    ref[:, 1] *= -1
    assert ((y - ref).abs() <= _i8_bound(ref)).all()


# ------------------------------------------------------------------------------------------------ gated projections

def _gated_reference(x, wg, wu, act):
    """h, g, u and what fp32 sums and a few roundings may be off by in h"""
    g, u = x @ wg.T, x @ wu.T
    dg, du = (2e-6 * (x.abs() @ w.abs().T) for w in (wg, wu))       # 2^-24 sqrt-like growth over k in fp32: 1e-5 is the linear tests' allowance for 5120
    a = _act(g, act)
    off = dg * 1.2 * u.abs() + a.abs() * du + 16 * 2.0 ** -24 * (a * u).abs()       # |act'| <= 1.13
    return a * u, g, u, off


def _kept(saved, M, F):
    """[2, M, F] of what training saves: blocks of 16 rows and 32 columns, of each the first four of every eight columns of all rows, then the others"""
    t = saved.view(2, -(-M // 16), -(-F // 32), 2, 4, 16, 4).permute(0, 1, 5, 2, 4, 3, 6)
    return t.reshape(2, -(-M // 16) * 16, -(-F // 32) * 32)[:, :M, :F]


GATED = [(1, 8, 128), (1, 1000, 640), (2, 72, 5120), (16, 64, 256), (17, 40, 128), (32, 136, 384), (33, 8, 128), (63, 128, 256), (65, 200, 128),
         (129, 72, 640), (300, 1032, 512), (1100, 1400, 256), (2050, 1160, 128), (2050, 2184, 384), (4680, 776, 256), (700, 4504, 384)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", GATED)
def test_gated_linear(M, F, K, act):
    from paper_2511_20426_amd.runner import gated_linear, gated_linear_train
    gen = _gen(M + F + K)
    x, wg, wu = _normal(gen, M + 1, K + 8), _normal(gen, F, K + 16, scale=2 * K ** -0.5), _normal(gen, F, K, scale=K ** -0.5)
    y = torch.full((M + 2, F + 24), 7.0, dtype=torch.bfloat16, device=DEV)
    gated_linear(x[:M, :K], wg[:, :K], wu, act, out=y[:M, :F])
    torch.cuda.synchronize()
    assert (y[M:] == 7).all() and (y[:, F:] == 7).all()
    h, g, u, off = _gated_reference(x[:M, :K].double().cpu(), wg[:, :K].double().cpu(), wu.double().cpu(), act)
    got = y[:M, :F].double().cpu()
    assert ((got - h).abs() <= h.abs() * 2.0 ** -8 + 1.05 * off + 1e-30).all()
    h2, saved = gated_linear_train(x[:M, :K], wg[:, :K], wu, act)
    assert (h2 == y[:M, :F]).all()
    kept = _kept(saved, M, F)
    for p, t in ((g, kept[0]), (u, kept[1])):
        w = wg[:, :K] if p is g else wu
        assert ((t.double().cpu() - p).abs() <= 2e-6 * (x[:M, :K].double().cpu().abs() @ w.double().cpu().abs().T)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 200])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gates_that_are_large(M, act):
    """Gates of 1e10 and -1e10 pass u or give zero, NaN and infinities stay in their rows."""
    from paper_2511_20426_amd.runner import gated_linear
    x, w = torch.zeros((M, 128), dtype=torch.bfloat16, device=DEV), torch.zeros((8, 128), dtype=torch.bfloat16, device=DEV)
    w[:, 0] = 1e10
    x[0, 0], x[1, 0], x[2, 0] = 1, -1, float("nan")
    wu = torch.zeros_like(w)
    wu[:, 0] = 2
    y = gated_linear(x, w, wu, act)
    big = torch.tensor(1e10, dtype=torch.bfloat16).double() * 2
    assert ((y[0].double().cpu() - big).abs() <= big * 2.0 ** -8).all() and (y[1] == 0).all() and y[2].isnan().all() and (y[3:] == 0).all()


def _gated_grads(x, wg, wu, dh, act):
    """Gradients, and how far bf16 roundings of dg and du take them"""
    g = (x @ wg.T).requires_grad_()
    u, e = x @ wu.T, 2.0 ** -8
    a = _act(g, act)
    slope = torch.autograd.grad(a.sum(), g)[0]
    a = a.detach()
    dg, du = dh * u * slope, dh * a
    ddg, ddu = e * dg.abs(), e * du.abs()
    out = []
    for ref, off, size in ((dg @ wg + du @ wu, ddg @ wg.abs() + ddu @ wu.abs(), dg.abs() @ wg.abs() + du.abs() @ wu.abs()),
                           (dg.T @ x, ddg.T @ x.abs(), dg.abs().T @ x.abs()), (du.T @ x, ddu.T @ x.abs(), du.abs().T @ x.abs())):
        out.append((ref, ref.abs() * e + off + 1e-5 * size + 1e-30))
    return out


GRADS = [(1, 8, 128), (4, 1000, 640), (5, 72, 256), (8, 520, 128), (9, 64, 384), (16, 2056, 256), (17, 40, 128), (64, 64, 128), (127, 136, 384), (128, 200, 128), (130, 1000, 640), (1000, 328, 256), (2345, 776, 384)]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", GRADS)
def test_gated_backward(M, F, K, act):
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen = _gen(M + F + K + 1)
    x, wg, wu = _normal(gen, M, K + 8)[:, :K], _normal(gen, F, K + 16, scale=2 * K ** -0.5)[:, :K], _normal(gen, F, K, scale=K ** -0.5)
    dh = _normal(gen, M, F + 8)[:, :F]
    _, saved = gated_linear_train(x, wg, wu, act)
    got = gated_linear_backward(dh, x, wg, wu, saved, act)
    xd, wgd, wud, dhd = (t.double().cpu() for t in (x, wg, wu, dh))
    refs = _gated_grads(xd, wgd, wud, dhd, act)
    for t, (ref, bound) in zip(got, refs):
        assert t.shape == ref.shape and ((t.double().cpu() - ref).abs() <= bound).all()
    # the formulas against differences of the forward, along a direction of each
    step = 1e-5
    for i, ref in enumerate(r for r, _ in refs):
        move = torch.randn(ref.shape, generator=gen, dtype=torch.float64)
        at = lambda sg: [t + sg * step * move if j == i else t for j, t in enumerate((xd, wgd, wud))]  # noqa: E731
        loss = lambda p: (dhd * _act(p[0] @ p[1].T, act) * (p[0] @ p[2].T)).sum()  # noqa: E731
        along = (loss(at(1)) - loss(at(-1))) / (2 * step)
        assert abs(along - (ref * move).sum()) <= 1e-6 * (ref * move).abs().sum() + 1e-6


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 100])
def test_gradients_that_are_asked_for(M):
    """Each of the three alone, and weights' gradients that do not lie one behind the other: the bits of all three together; what is not asked
    for is not written."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen, F, K = _gen(M), 72, 256
    x, wg, wu, dh = _normal(gen, M, K), _normal(gen, F, K), _normal(gen, F, K), _normal(gen, M, F)
    _, saved = gated_linear_train(x, wg, wu)
    whole = gated_linear_backward(dh, x, wg, wu, saved)
    nbytes = B.layer_gated_backward_workspace(M, F, K)
    work = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    for asked in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 1)):
        out = [torch.full((n + 2, K + 8), 7.0, dtype=torch.bfloat16, device=DEV) for n in (M, F, F)]
        B.layer_gated_backward_bf16(dh.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), saved.data_ptr(), B.CA_SILU,
                                    *(t.data_ptr() if a else 0 for t, a in zip(out, asked)), M, F, K, F, K, K, K, K + 8, K + 8, work.data_ptr(), nbytes,
                                    torch.cuda.current_stream().cuda_stream)
        for t, ref, a in zip(out, whole, asked):
            n = ref.shape[0]
            assert (t[:n, :K] == ref).all() if a else (t[:n, :K] == 7).all()
            assert (t[n:] == 7).all() and (t[:, K:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 100])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradients_of_gates_that_are_nan(M, act):
    """A NaN among the gate's weights is in the gradients of both weights of its column and of all rows, and in no other column's."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen = _gen(21)
    x, wg, wu, dh = _normal(gen, M, 128), _normal(gen, 16, 128), _normal(gen, 16, 128), _normal(gen, M, 16)
    wg[5, 0] = float("nan")
    _, saved = gated_linear_train(x, wg, wu, act)
    dx, dwg, dwu = gated_linear_backward(dh, x, wg, wu, saved, act)
    bad = torch.arange(16, device=DEV) == 5
    for t in (dwg, dwu):
        assert t[bad].isnan().all() and t[~bad].isfinite().all()
    assert dx.isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,F,K", [(5, 8, 128), (7, 136, 128), (11, 2000, 5120), (16, 264, 1664), (20, 72, 384), (31, 4008, 640), (32, 2056, 2560), (33, 136, 256)])
def test_gradients_of_some_rows(M, F, K):
    """Up to 32 rows: several chunks of columns, ends inside a chunk and a wave's part, strided weights; then each of the three alone and into
    strides, with the bits of all together, and nothing beside them written."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen = _gen(M + F + K + 7)
    x, wg, wu = _normal(gen, M, K + 24)[:, :K], _normal(gen, F, K + 8, scale=2 * K ** -0.5)[:, :K], _normal(gen, F, K, scale=K ** -0.5)
    dh = _normal(gen, M, F + 16)[:, :F]
    _, saved = gated_linear_train(x, wg, wu, "gelu")
    whole = gated_linear_backward(dh, x, wg, wu, saved, "gelu")
    for t, (ref, bound) in zip(whole, _gated_grads(*(t.double().cpu() for t in (x, wg, wu, dh)), "gelu")):
        assert ((t.double().cpu() - ref).abs() <= bound).all()
    nbytes = B.layer_gated_backward_workspace(M, F, K)
    work = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    for asked in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 1)):
        out = [torch.full((n + 2, K + 8), 7.0, dtype=torch.bfloat16, device=DEV) for n in (M, F, F)]
        B.layer_gated_backward_bf16(dh.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), saved.data_ptr(), B.CA_GELU,
                                    *(t.data_ptr() if a else 0 for t, a in zip(out, asked)), M, F, K, F + 16, K + 24, K + 8, K, K + 8, K + 8, work.data_ptr(),
                                    nbytes, torch.cuda.current_stream().cuda_stream)
        for t, ref, a in zip(out, whole, asked):
            n = ref.shape[0]
            assert (t[:n, :K] == ref).all() if a else (t[:n, :K] == 7).all()
            assert (t[n:] == 7).all() and (t[:, K:] == 7).all()


@pytest.mark.gpu
def test_gated_of_no_rows():
    from paper_2511_20426_amd.runner import gated_linear, gated_linear_backward, gated_linear_train
    x, w = torch.empty((0, 128), dtype=torch.bfloat16, device=DEV), torch.ones((16, 128), dtype=torch.bfloat16, device=DEV)
    assert gated_linear(x, w, w).shape == (0, 16)
    h, saved = gated_linear_train(x, w, w)
    dx, dwg, dwu = gated_linear_backward(h, x, w, w, saved)
    assert dx.shape == (0, 128) and (dwg == 0).all() and (dwu == 0).all()


# ------------------------------------------------------------------------------------------------ all of them

@pytest.mark.gpu
def test_offsets_that_pass_32_bits():
    """Operands and results of more than 2^31 values: the last rows against the same rows alone."""
    from paper_2511_20426_amd.runner import gated_linear, gated_linear_train, linear_i8, quantize_rows
    gen = torch.Generator(device=DEV).manual_seed(2)
    pool = _pool(40, 128, (30, 52))
    n = 140013
    qkv = torch.randn((n, 3, 40, 128), generator=gen, device=DEV, dtype=torch.bfloat16)      # 2.15e9 values
    w = torch.ones(128, dtype=torch.bfloat16, device=DEV)
    k = pool.qk_norm_rope(None, qkv[:, 1], None, w, 0, k_out=qkv[:, 2])[1]
    first = 89                                    # (a frame has 1560 tokens)
    alone = pool.qk_norm_rope(None, qkv[1560 * first:, 1], None, w, first)[1]
    assert (k[1560 * first:] == alone).all()
    del qkv, k, alone
    M, N = 140001, 15360
    x = torch.randn((M, 128), generator=gen, device=DEV, dtype=torch.bfloat16)
    wn = quantize_rows(torch.randn((N, 128), generator=gen, device=DEV, dtype=torch.bfloat16))
    y = linear_i8(x, wn)
    assert (y[-300:] == linear_i8(x[-300:], wn)).all() and (y[:300] == linear_i8(x[:300], wn)).all()
    del y
    wg, wu = (torch.randn((N, 128), generator=gen, device=DEV, dtype=torch.bfloat16) / 11 for _ in range(2))
    h, saved = gated_linear_train(x, wg, wu)
    assert (h[-300:] == gated_linear(x[-300:], wg, wu)).all()
    few, kept = gated_linear_train(x[-300:], wg, wu)
    assert (few == h[-300:]).all()
    assert (_kept(saved, M, N)[:, -300:] == _kept(kept, 300, N)).all()


@pytest.mark.gpu
def test_replayed_from_a_graph():
    """All calls recorded once and replayed with other inputs, between eager work: every replay gives the eager calls' bits."""
    from paper_2511_20426_amd import runner as R
    pool, gen = _pool(2, 128, (4, 5)), _gen(9)
    n, K, F = 120, 256, 264
    qkv, dz, w = _normal(gen, n, 3, 2, 128), _normal(gen, n, 2, 2, 128), _normal(gen, 128)
    x, wg, wu, dh = _normal(gen, n, K), _normal(gen, F, K), _normal(gen, F, K), _normal(gen, n, F)
    wq = R.quantize_rows(_normal(gen, 64, K))

    def calls():
        out = list(pool.qk_norm_rope(qkv[:, 0], qkv[:, 1], w, w, 3))
        out += pool.qk_norm_rope_backward(dz[:, :, 0], dz[:, :, 1], qkv[:, 0], qkv[:, 1], w, w, 3)
        out += [R.linear_i8(x, wq), R.linear_i8(x[:5], wq)]
        h, saved = R.gated_linear_train(x, wg, wu, "gelu")
        return out + [h, R.gated_linear(x[:3], wg, wu), *R.gated_linear_backward(dh, x, wg, wu, saved, "gelu")]

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = calls()
    for i in range(4):
        for t in (qkv, dz, x, dh):
            t.copy_(torch.randn(t.shape, generator=gen).to(t.dtype))
        eager = calls()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all((a == b).all() for a, b in zip(held, eager)), i


@pytest.mark.gpu
def test_both_ways_do_the_same(monkeypatch):
    """The calls that the extension takes and those that go through the Python code give the same bits, given results or none."""
    from paper_2511_20426_amd import runner as R
    pool, gen = _pool(2, 128, (4, 5)), _gen(12)
    n, K, F = 60, 256, 136
    qkv, dz, w = _normal(gen, n, 3, 2, 128), _normal(gen, n, 2, 2, 128), _normal(gen, 128)
    x, wg, wu, dh = _normal(gen, n, K), _normal(gen, F, K), _normal(gen, F, K), _normal(gen, n, F)
    wq = R.quantize_rows(_normal(gen, 64, K))

    def results():
        new = lambda t: torch.empty(t.shape, dtype=t.dtype, device=DEV)  # noqa: E731
        q, k = new(qkv[:, 0]), new(qkv[:, 1])
        assert pool.qk_norm_rope(qkv[:, 0], qkv[:, 1], w, w, 3, q_out=q, k_out=k)[1] is k
        out = [q, k, *pool.qk_norm_rope(qkv[:, 0], None, w, None, 3)[:1], *pool.qk_norm_rope(None, qkv[:1, 1], None, w, 3)[1:]]
        out += pool.qk_norm_rope_backward(dz[:, :, 0], dz[:, :, 1], qkv[:, 0], qkv[:, 1], w, w, 3)
        dk = dz[:, :, 1].clone()
        some = pool.qk_norm_rope_backward(None, dk, None, qkv[:, 1], None, w, 3, dk=dk)
        assert some[0] is None and some[1] is dk and some[2] is None
        out += [dk, some[3]]
        assert pool.append_batch([1], [0], 0, [qkv[:, 1]], [qkv[:, 2]], k_weight=w) == [1]
        at = pool.ctx.kv_cache_page_index(1, 0, 0) * 65536
        out.append(pool.pool[at:at + 2 * 65536].clone())
        y, h = torch.empty((n, 64), dtype=torch.bfloat16, device=DEV), torch.empty((n, F + 8), dtype=torch.bfloat16, device=DEV)[:, :F]
        assert R.linear_i8(x, wq, out=y) is y
        out += [y, R.linear_i8(x[:1], wq), R.linear_i8(x.float(), wq), R.linear_i8(R.quantize_rows(x), wq)]
        assert R.gated_linear(x, wg, wu, out=h) is h
        h2, saved = R.gated_linear_train(x, wg, wu, "gelu")
        return out + [h, R.gated_linear(x[:1], wg, wu), h2, _kept(saved, n, F), *R.gated_linear_backward(dh, x, wg, wu, saved, "gelu")]

    first = results()
    monkeypatch.setattr(B, "calls", B._NoCalls())
    second = results()
    assert len(first) == len(second)
    for i, (a, b) in enumerate(zip(first, second)):
        assert a.shape == b.shape and a.dtype == b.dtype and (a == b).all(), i
    assert (first[11] == first[14]).all()         # codes made on the way or before


def _refused(code, call, *args):
    with pytest.raises(B.CascadeAttnError) as e:
        call(*args)
    assert e.value.code == code, (args, e.value)


def test_refusals():
    """What the shapes, strides and pointers rule out is refused before anything is launched (no GPU is needed to be refused)."""
    cfg = B.make_config(heads=2, head_dim=128, frames_per_block=3, grid_h=4, grid_w=5, rope_dims=ROPE[128], rope_theta=1e4, sink_blocks=0,
                        window_blocks=2, max_inflight=2, page_tokens=128, dtype="bf16")
    ctx = B.Context(cfg)
    t = (4096, 256, 128)
    _refused(B.CA_ENOPOOL, ctx.layer_qk_norm_rope, t, t, 16, 16, 1e-6, t, t, 4, 0)
    _refused(B.CA_ENOPOOL, ctx.kv_cache_append_batch_norm, [0], [0], 0, [16], [16], 256, 128, 16, 1e-6)
    _refused(B.CA_ENOPOOL, ctx.layer_qk_norm_rope_backward, t, t, t, t, 16, 16, 1e-6, t, t, 16, 16, 4, 0, 4096, 1 << 30)
    # a context over an address that no call below gets to use
    nbytes = B.pool_bytes(cfg)
    ctx = B.Context(cfg, 1 << 40, nbytes)
    ok = [t, t, 16, 16, 1e-6, t, t, 4, 0]
    for i, bad in [(0, (4096, 256, 64)), (0, (4096, 100, 128)), (0, (4096, 252, 128)), (0, (4098, 256, 128)), (0, (0, 256, 128)), (1, (4096, -256, 128)),
                   (2, 0), (2, 24), (3, None), (4, -1.0), (4, float("nan")), (4, float("inf")), (5, None), (6, (4096, 0, 128)), (7, -1), (8, -1)]:
        args = list(ok)
        args[i] = bad
        _refused(B.CA_EINVAL, ctx.layer_qk_norm_rope, *args)
    for n, first in ((1 << 31, 0), (4, 1 << 31), (1 << 30, (1 << 30) + 8)):
        _refused(B.CA_EUNSUPPORTED, ctx.layer_qk_norm_rope, *ok[:7], n, first)
    _refused(B.CA_EUNSUPPORTED, ctx.kv_cache_append_batch_norm, [1 << 40], [0], 0, [4096], [4096], 256, 128, 16, 1e-6)
    _refused(B.CA_EINVAL, ctx.layer_qk_norm_rope, None, None, 0, 0, 1e-6, None, None, 4, 0)
    _refused(B.CA_EINVAL, ctx.layer_qk_norm_rope, None, t, 0, 16, 1e-6, t, t, 4, 0)
    need = ctx.layer_qk_norm_rope_workspace()
    ok = [t, t, t, t, 16, 16, 1e-6, t, t, 16, 16, 4, 0, 4096, need]
    for i, bad in [(0, None), (1, (0, 256, 128)), (2, (4096, 255, 128)), (4, None), (6, -1e-6), (7, None), (9, 0), (10, None), (11, -1), (13, 0), (13, 8), (14, need - 1)]:
        args = list(ok)
        args[i] = bad
        _refused(B.CA_EINVAL, ctx.layer_qk_norm_rope_backward, *args)
    ok = [[0], [0], 0, [4096], [4096], 256, 128, 16, 1e-6]
    for i, bad, code in [(0, [-1], B.CA_EINVAL), (3, [0], B.CA_EINVAL), (4, [8], B.CA_EINVAL), (5, 255, B.CA_EINVAL), (7, 0, B.CA_EINVAL), (7, 8, B.CA_EINVAL),
                         (8, -1.0, B.CA_EINVAL)]:
        args = list(ok)
        args[i] = bad
        _refused(code, ctx.kv_cache_append_batch_norm, *args)
    _refused(B.CA_EINVAL, ctx.kv_cache_append_batch_norm, [0, 0], [0, 0], 0, [4096] * 2, [4096] * 2, 256, 128, 16, 1e-6)
    _refused(B.CA_ENOSPC, ctx.kv_cache_append_batch_norm, [0, 4], [0, 0], 0, [4096] * 2, [4096] * 2, 256, 128, 16, 1e-6)
    assert ctx.kv_cache_snapshot() == []

    E, U = B.CA_EINVAL, B.CA_EUNSUPPORTED
    ok = [4096, B.CA_BF16, 4096, 4096, 5, 300, 300, 512]
    for i, bad, code in [(0, 0, E), (0, 4097, E), (1, 2, E), (2, 0, E), (2, 4104, E), (3, 0, E), (3, 4098, E), (4, -1, E), (4, 1 << 31, U), (5, 0, U),
                         (5, B.CA_I8_MAX_K + 1, U), (6, 299, E), (7, 511, E), (7, 256, E)]:
        args = list(ok)
        args[i] = bad
        _refused(code, B.layer_quantize_rows_i8, *args)
    ok = [4096] * 5 + [5, 16, 300, 512, 512, 16]
    for i, bad, code in [(0, 0, E), (1, 0, E), (2, 4104, E), (3, 4100, E), (4, 0, E), (4, 4104, E), (5, -1, E), (5, 1 << 31, U), (6, 12, U), (6, 0, U), (7, 0, U),
                         (7, B.CA_I8_MAX_K + 1, U), (8, 256, E), (8, 520, E), (9, 504, E), (9, 1 << 24, U), (10, 8, E), (10, 20, E)]:
        args = list(ok)
        args[i] = bad
        _refused(code, B.layer_linear_i8, *args)
    need = B.layer_linear_i8_workspace(5, 300)
    assert need >= 5 * (512 + 4) and B.layer_linear_i8_workspace(5, 0) == 0 == B.layer_linear_i8_workspace(-1, 8)
    ok = [4096, B.CA_BF16, 4096, 4096, 4096, 5, 16, 300, 300, 512, 16, 4096, need]
    for i, bad, code in [(0, 0, E), (0, 4097, E), (1, 7, E), (2, 4104, E), (3, 4100, E), (4, 0, E), (5, -1, E), (6, 4, U), (7, 0, U), (8, 299, E), (8, 1 << 22, U), (9, 256, E),
                         (10, 12, E), (11, 0, E), (11, 4104, E), (12, need - 1, E)]:
        args = list(ok)
        args[i] = bad
        _refused(code, B.layer_linear_i8_values, *args)
    assert B.layer_gated_saved_bytes(5, 40) == 2 * 16 * 64 * 4 and B.layer_gated_saved_bytes(5, 4) == 0
    ok = [4096] * 5 + [B.CA_SILU, 5, 16, 128, 128, 128, 128, 16]
    for i, bad, code in [(0, 0, E), (1, 4104, E), (2, 0, E), (3, 0, E), (4, 8, E), (5, 2, E), (6, -1, E), (6, 1 << 31, U), (7, 12, U), (8, 64, U), (8, 192, U),
                         (9, 120, E), (10, 132, E), (11, 1 << 22, U), (12, 8, E)]:
        args = list(ok)
        args[i] = bad
        _refused(code, B.layer_gated_bf16, *args)
    need = B.layer_gated_backward_workspace(5, 16, 128)
    assert need > 0 and B.layer_gated_backward_workspace(5, 12, 128) == 0 == B.layer_gated_backward_workspace(-1, 16, 128)
    ok = [4096] * 5 + [B.CA_GELU] + [4096] * 3 + [5, 16, 128, 16, 128, 128, 128, 128, 128, 4096, need]
    for i, bad, code in [(0, 0, E), (1, 0, E), (2, 0, E), (3, 4104, E), (4, 0, E), (5, -1, E), (6, 8, E), (9, -1, E), (9, 1 << 23, U), (10, 4, U), (11, 100, U),
                         (12, 8, E), (13, 120, E), (16, 127, E), (17, 1 << 22, U), (18, 0, E), (18, 4104, E), (19, need - 1, E)]:
        args = list(ok)
        args[i] = bad
        _refused(code, B.layer_gated_backward_bf16, *args)
    _refused(E, B.layer_gated_backward_bf16, *ok[:6], 0, 0, 0, *ok[9:])


def test_workspaces_of_refused_shapes():
    """The backward pass's workspace is 0 bytes for shapes that the call refuses, those whose row strides are too long among them."""
    most = (1 << 22) - 256
    assert B.layer_gated_backward_workspace(most, 16, 128) > 0
    for m, f, k in ((most + 1, 16, 128), (1 << 30, 16, 128), (5, (1 << 21) - 56, 128), (1 << 30, 2**31 - 8, 128), (5, 16, 1 << 22)):
        assert B.layer_gated_backward_workspace(m, f, k) == 0
        ldf, ldk = -(-f // 8) * 8, k
        code = B.CA_EUNSUPPORTED
        _refused(code, B.layer_gated_backward_bf16, *[4096] * 5, B.CA_SILU, *[4096] * 3, m, f, k, ldf, ldk, ldk, ldk, ldk, ldk, 4096, 1 << 62)


def test_launches_that_are_too_large_are_refused():
    """Sizes whose launch would have 2^32 threads."""
    cfg = B.make_config(heads=2, head_dim=128, frames_per_block=3, grid_h=4, grid_w=5, rope_dims=ROPE[128], rope_theta=1e4, sink_blocks=0,
                        window_blocks=2, max_inflight=2, page_tokens=128, dtype="bf16")
    ctx, t = B.Context(cfg, 1 << 40, B.pool_bytes(cfg)), (4096, 256, 128)
    _refused(B.CA_EUNSUPPORTED, ctx.layer_qk_norm_rope, t, t, 16, 16, 1e-6, t, t, 1 << 26, 0)
    for rows, k in ((1 << 24, 4096), (1 << 26, 8)):
        _refused(B.CA_EUNSUPPORTED, B.layer_quantize_rows_i8, 4096, B.CA_BF16, 4096, 4096, rows, k, k, -(-k // 256) * 256)


@pytest.mark.parametrize("host", [b"bytes of the host", (C.c_char * 64)(), 16.0, np.int64(16)], ids=["bytes", "array", "float", "numpy"])
def test_addresses_are_integers(host):
    calls = [(B.layer_quantize_rows_i8, [16, 1, 16, 16, 0, 8, 8, 256], (0, 2, 3)), (B.layer_linear_i8, [16] * 5 + [0, 8, 8, 256, 256, 8], range(5)),
             (B.layer_linear_i8_values, [16, 1, 16, 16, 16, 0, 8, 8, 8, 256, 8, 16, 1 << 20], (0, 2, 3, 4, 11)),
             (B.layer_gated_bf16, [16] * 5 + [0, 0, 8, 128, 128, 128, 128, 8], range(5)),
             (B.layer_gated_backward_bf16, [16] * 5 + [0] + [16] * 3 + [0, 8, 128, 8, 128, 128, 128, 128, 128, 16, 0], (0, 1, 2, 3, 4, 6, 7, 8, 18))]
    for call, args, pointers in calls:
        for i in pointers:
            with pytest.raises(TypeError):
                call(*[host if j == i else a for j, a in enumerate(args)])


@pytest.mark.gpu
def test_refusals_of_the_torch_calls():
    from paper_2511_20426_amd import runner as R
    pool, t = _pool(2), dict(dtype=torch.bfloat16, device=DEV)
    q, w = torch.zeros((6, 2, 128), **t), torch.ones(128, **t)
    for bad in (lambda: pool.qk_norm_rope(q.float(), None, w, None, 0), lambda: pool.qk_norm_rope(q, None, w.float(), None, 0),
                lambda: pool.qk_norm_rope(q, q[:5], w, w, 0), lambda: pool.qk_norm_rope(q, None, w, None, 0, q_out=q.float()),
                lambda: pool.qk_norm_rope(q, None, w[:64], None, 0), lambda: pool.qk_norm_rope(q, None, w, w, 0),
                lambda: pool.qk_norm_rope_backward(None, None, q, None, w, None, 0), lambda: pool.qk_norm_rope(q.cpu(), None, w, None, 0)):
        with pytest.raises((AssertionError, AttributeError)):
            bad()
    x, m = torch.zeros((4, 128), **t), torch.zeros((16, 128), **t)
    wq = R.quantize_rows(m)
    for bad in (lambda: R.quantize_rows(x.half()), lambda: R.quantize_rows(x.cpu()), lambda: R.linear_i8(x[:, :64], wq),
                lambda: R.linear_i8(x, wq, out=torch.zeros((4, 16), device=DEV)), lambda: R.linear_i8(x, wq, out=torch.zeros((4, 8), **t)),
                lambda: R.gated_linear(x, m, m[:8]), lambda: R.gated_linear(x.T, m, m), lambda: R.gated_linear(x, m, m.float()),
                lambda: R.gated_linear(x, m, m, out=torch.zeros((4, 16))), lambda: R.gated_linear_backward(x, x, m, m, torch.zeros((2, 4, 16), device=DEV))):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(KeyError):
        R.gated_linear(x, m, m, "relu")


# ------------------------------------------------------------------------------------------------ a layer of them

def _in_8_bits(t):
    """what the codes of t's rows stand for"""
    most = t.abs().amax(1, keepdim=True)
    return torch.round(t * 127 / torch.where(most > 0, most, 1.0)) * most / 127


@pytest.mark.gpu
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_layer(activation):
    """A layer's iteration against the same in 64 bits from its own 8-bit weights: two cached blocks, two in flight, an odd grid."""
    from paper_2511_20426_amd.layer import CascadeLayer
    gen, heads, grid, F, D = _gen(21), 2, (5, 7), 328, 128
    width, L = heads * D, 105
    pool = _pool(heads, D, grid)
    ws = [_normal(gen, *s, scale=s[1] ** -0.5) for s in ((3 * width, width), (width, width), (F, width), (F, width), (width, F))]
    norms = [_normal(gen, D) for _ in range(2)]
    layer = CascadeLayer.from_weights(*ws, *norms, activation=activation)
    cached = [(_normal(gen, L, heads, D), _normal(gen, L, heads, D)) for _ in range(2)]
    for g, (k, v) in enumerate(cached):
        pool.append(g, 0, 0, k, v)
        pool.ctx.kv_cache_promote(g)
    x = _normal(gen, 2 * L, width)
    got = layer(pool, x, [2, 3], [500, 1000], mode=B.CA_BLOCK_CAUSAL).double().cpu()

    wqkv, wo, wg, wu, wd = (w.double().cpu() for w in ws)
    linear8 = lambda t, w: _in_8_bits(t) @ _in_8_bits(w).T  # noqa: E731
    x = x.double().cpu()
    qkv = linear8(x, wqkv).view(2 * L, 3, heads, D)
    ang = _angles(D, grid, 6, 2 * L)
    q, k = (_norm_rope(qkv[:, s], n.double().cpu(), 1e-6, ang).transpose(0, 1) for s, n in zip((0, 1), norms))
    ks = torch.cat([_rotate(k_.double().cpu(), _angles(D, grid, 3 * g, L)).transpose(0, 1) for g, (k_, _) in enumerate(cached)] + [k], 1)
    vs = torch.cat([v_.double().cpu().transpose(0, 1) for _, v_ in cached] + [qkv[:, 2].transpose(0, 1)], 1)
    logits = q @ ks.transpose(1, 2) / D ** 0.5
    logits[:, :L, 3 * L:] = -torch.inf             # the first block in flight does not see the second
    o = (torch.softmax(logits, -1) @ vs).transpose(0, 1).reshape(2 * L, width)
    y = x + linear8(o, wo)
    ref = y + linear8(_act(y @ wg.T, activation) * (y @ wu.T), wd)
    # roundings to bf16 on the way (2^-8 each, at most 8 of them between x and the result) and 8-bit codes that fall on the other side of a border
    # for them (a step is 1/127 of a row's largest value, a few in a thousand of the codes): 2 % of the norm
    assert (got - ref).norm() <= 2e-2 * ref.norm()


@pytest.mark.gpu
def test_feed_forward_training():
    """Gradients of a step against 64 bits, and that steps lead down."""
    from paper_2511_20426_amd.layer import feed_forward_step
    gen = _gen(22)
    M, K, F = 200, 128, 136 * 128 // 8
    x, wg, wu, wd = _normal(gen, M, K), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, K, F, scale=F ** -0.5)
    target = _normal(gen, M, K)
    leaves = [t.double().cpu().requires_grad_() for t in (wg, wu, wd, x)]
    loss = ((_act(leaves[3] @ leaves[0].T, "silu") * (leaves[3] @ leaves[1].T) @ leaves[2].T - target.double().cpu()) ** 2).mean()
    refs = torch.autograd.grad(loss, leaves)
    got, grads = feed_forward_step(x, wg, wu, wd, target)
    assert abs(got.item() - loss.item()) <= 2e-2 * loss.item()
    for g, r in zip(grads, refs):                  # at most five bf16 roundings on the way to each: 5 * 2^-8
        assert (g.double().cpu() - r).norm() <= 2e-2 * r.norm()
    losses = [feed_forward_step(x, wg, wu, wd, target, lr=2.0)[0].item() for _ in range(8)]
    assert losses[-1] < losses[0] - 1e-3


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    import os
    import shutil
    import subprocess
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc, exe = os.path.join(root, "paper_2511_20426_amd", "csrc"), str(tmp_path / "layer_sanitize")
    subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
                    "-I", os.path.join(root, "include"), "-I", csrc, os.path.join(root, "tests", "layer_sanitize_driver.cpp")] +
                   [os.path.join(csrc, f) for f in ("ca_layer.cpp", "ca_api.cpp", "ca_meta.cpp")] + ["-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
                                                                                 UBSAN_OPTIONS="print_stacktrace=1"))
    assert r.returncode == 0 and "layer sanitizer driver: ok" in r.stdout, r.stdout + r.stderr
