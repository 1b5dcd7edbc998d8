"""The operators around the attention where they could go wrong and tests/test_layer_ops.py does not look: values that are not finite in the
last rows of weights, products walked in parts, the precision that each number of rows has, and calls that must not reach a kernel."""
import pytest
import torch

from paper_2511_20426_amd import binding as B
from tests.test_layer_ops import DEV, HALF, WAY, _act, _angles, _gated_grads, _gen, _kept, _norm_grads, _norm_rope, _normal, _pairs, _pool


def _given_gradients(g, u, dh, act):
    """dg and du of saved projections, in 64 bits"""
    g = g.double().requires_grad_()
    a = _act(g, act)
    slope = torch.autograd.grad(a.sum(), g)[0]
    return dh * u.double() * slope, dh * a.detach()


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["gate", "up"])
@pytest.mark.parametrize("F", [72, 136, 256])
@pytest.mark.parametrize("M", [3, 4, 5, 8, 16, 17, 20, 32, 40])
def test_an_infinity_in_the_last_row_of_weights(M, F, which):
    """... is an infinity in its column of dX, of the sign of its gradient, and nowhere else, for any number of rows and of columns f."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen, K = _gen(M + F), 128
    x, wg, wu, dh = _normal(gen, M, K), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, M, F)
    _, saved = gated_linear_train(x, wg, wu)
    xd, gd, ud = (t.double().cpu() for t in (x, wg, wu))
    dg, du = _given_gradients(xd @ gd.T, xd @ ud.T, dh.double().cpu(), "silu")
    (wg if which == "gate" else wu)[F - 1, 5] = float("inf")
    dx, dwg, dwu = (t.double().cpu() for t in gated_linear_backward(dh, x, wg, wu, saved))
    d = (dg if which == "gate" else du)[:, F - 1]
    assert (d != 0).all() and (dx[:, 5] == d.sign() * float("inf")).all()
    dx[:, 5] = 0
    assert all(t.isfinite().all() for t in (dx, dwg, dwu))


def _given_saved(M, F, K, act, seed):
    """inputs of a backward pass and dg, du of the projections that it is given, in 64 bits"""
    from paper_2511_20426_amd.runner import gated_linear_train
    gen = _gen(seed)
    x, wg, wu, dh = _normal(gen, M, K), _normal(gen, F, K, scale=2 * K ** -0.5), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, M, F)
    _, saved = gated_linear_train(x, wg, wu, act)
    g, u = (t.double().cpu() for t in _kept(saved, M, F))
    return x, wg, wu, dh, saved, g, u


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", [(1, 8, 128), (4, 72, 256), (4, 200, 128), (5, 8, 128), (5, 64, 256), (8, 136, 128), (9, 264, 128), (16, 40, 384), (17, 8, 128),
                                   (24, 200, 256), (32, 64, 128), (32, 392, 128)])
def test_gradients_of_few_rows_keep_their_bits(M, F, K, act):
    """Of up to four rows dg and du go into the products in fp32, of 5 to 32 as two bf16 values each: within 2^-15 of themselves."""
    from paper_2511_20426_amd.runner import gated_linear_backward
    x, wg, wu, dh, saved, g, u = _given_saved(M, F, K, act, M + F + K)
    dg, du = _given_gradients(g, u, dh.double().cpu(), act)
    # in fp32: some 16 roundings of 2^-24 and the exponent's (p 2^-23, |p| < 64 at these gates) of terms of the size of dh u and of du; the cut and
    # rest of a value: the rest is below 2^-7 of it and half a step, 2^-8, off
    cut = 2.0 ** -15 if M > 4 else 0.0
    ddg, ddu = 2.0 ** -17 * (dh.double().cpu() * u).abs() + cut * dg.abs(), (2.0 ** -17 + cut) * du.abs()
    xd, gd, ud = (t.double().cpu() for t in (x, wg, wu))
    refs = ((dg @ gd + du @ ud, ddg @ gd.abs() + ddu @ ud.abs(), dg.abs() @ gd.abs() + du.abs() @ ud.abs()),
            (dg.T @ xd, ddg.T @ xd.abs(), dg.abs().T @ xd.abs()), (du.T @ xd, ddu.T @ xd.abs(), du.abs().T @ xd.abs()))
    for t, (ref, off, size) in zip(gated_linear_backward(dh, x, wg, wu, saved, act), refs):
        # one rounding of the result, fp32 sums of at most 784 products (1e-5 is the linear maps' allowance for 5120)
        assert ((t.double().cpu() - ref).abs() <= ref.abs() * 2.0 ** -8 + off + 1e-5 * size + 1e-30).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 8, 20, 40])
def test_infinities_meet_gradients_that_bf16_holds(M):
    """dg of 1/2, 2 and the like, which leave no rest: infinite weights and activations give infinities of their sign, not NaN; gradients of zero give
    NaN with them, as the formula does."""
    from paper_2511_20426_amd.runner import gated_linear_backward
    F, K = 24, 128
    dh = torch.tensor([1.0, -4.0, 0.25], device=DEV, dtype=torch.bfloat16)[torch.arange(M * F, device=DEV) % 3].view(M, F).contiguous()
    dh[:, 7] = 0
    half = B.layer_gated_saved_bytes(M, F) // 8
    saved = torch.cat((torch.zeros(half, device=DEV), torch.ones(half, device=DEV)))         # g = 0, u = 1: dg = dh / 2, du = 0
    gen = _gen(M)
    x, wg, wu = _normal(gen, M, K), _normal(gen, F, K), _normal(gen, F, K)
    x[1, 9], wg[3, 5], wg[4, 6], wg[7, 8] = float("inf"), float("inf"), float("-inf"), float("inf")
    dx, dwg, dwu = (t.double().cpu() for t in gated_linear_backward(dh, x, wg, wu, saved))
    d, inf = dh.double().cpu(), float("inf")
    assert (dx[:, 5] == d[:, 3].sign() * inf).all() and (dx[:, 6] == d[:, 4].sign() * -inf).all() and dx[:, 8].isnan().all()
    keep = torch.ones(F, dtype=torch.bool)
    keep[7] = False
    assert (dwg[keep, 9] == d[1, keep].sign() * inf).all() and dwg[7, 9].isnan() and dwu[:, 9].isnan().all()
    for t, cols in ((dx, [5, 6, 8]), (dwg, [9]), (dwu, [9])):
        t[:, cols] = 0
        assert t.isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 8, 20, 40])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_gradients_from_above_that_are_not_finite(M, value):
    """... reach the rows of dX and the columns f of the weights' gradients that they belong to, and no others."""
    from paper_2511_20426_amd.runner import gated_linear_backward
    F, K = 136, 128
    x, wg, wu, dh, saved, g, u = _given_saved(M, F, K, "silu", 5)
    dh[2, 131] = value
    dg, du = _given_gradients(g, u, dh.double().cpu(), "silu")
    dx, dwg, dwu = (t.double().cpu() for t in gated_linear_backward(dh, x, wg, wu, saved))
    rows, cols = torch.arange(M) == 2, torch.arange(F) == 131
    assert dx[~rows].isfinite().all() and not dx[rows].isfinite().any()
    for t, d in ((dwg, dg), (dwu, du)):
        ref = d[2, 131] * x[2].double().cpu()
        assert t[~cols].isfinite().all() and (t[cols][0].isnan() if value != value else t[cols][0] == ref).all()


def _parts_bytes(M, F, K):
    """what the workspace has behind the layout: room for the sums of products that are walked in parts"""
    up = lambda n, to: -(-n // to) * to  # noqa: E731
    rows, cols = up(M, 128), up(F, 64)
    return B.layer_gated_backward_workspace(M, F, K) - sum(up(2 * n, 256) for n in (M * 2 * cols, 2 * F * rows, K * rows, K * 2 * cols))


# dX in 8, 14 and 4 parts, weights' gradients in 11 and 6 (a last part that is shorter among them), rows and columns that
# end inside a tile (asserted, so that another model does not drop them)
IN_PARTS = [(100, 2000, 128), (65, 4008, 256), (4000, 40, 128), (3325, 64, 256), (777, 3000, 128)]


@pytest.mark.parametrize("M,F,K", IN_PARTS)
def test_which_products_are_walked_in_parts(M, F, K):
    assert _parts_bytes(M, F, K) > 0
    assert _parts_bytes(130, 1000, 640) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,F,K", IN_PARTS)
def test_gradients_by_products_in_parts(M, F, K, act):
    """Element by element; then each of the three alone, both weights' apart (their parts take the same room, one after the other), into strides:
    dX has the same bits, the weights' (which may be walked in other parts than as one product) the same bounds; nothing beside them is written."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen = _gen(M + F + K)
    x, wg, wu = _normal(gen, M, K + 8)[:, :K], _normal(gen, F, K + 16, scale=2 * K ** -0.5)[:, :K], _normal(gen, F, K, scale=K ** -0.5)
    dh = _normal(gen, M, F + 8)[:, :F]
    _, saved = gated_linear_train(x, wg, wu, act)
    whole = gated_linear_backward(dh, x, wg, wu, saved, act)
    refs = _gated_grads(*(t.double().cpu() for t in (x, wg, wu, dh)), act)
    for t, (ref, bound) in zip(whole, refs):
        assert ((t.double().cpu() - ref).abs() <= bound).all()
    nbytes = B.layer_gated_backward_workspace(M, F, K)
    work = torch.empty(nbytes + 4096, dtype=torch.uint8, device=DEV)
    for asked in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (1, 1, 1)):
        out = [torch.full((n + 2, K + 8), 7.0, dtype=torch.bfloat16, device=DEV) for n in (M, F, F)]
        work.fill_(0x55)
        B.layer_gated_backward_bf16(dh.data_ptr(), x.data_ptr(), wg.data_ptr(), wu.data_ptr(), saved.data_ptr(), B.CA_GELU if act == "gelu" else B.CA_SILU,
                                    *(t.data_ptr() if a else 0 for t, a in zip(out, asked)), M, F, K, F + 8, K + 8, K + 16, K, K + 8, K + 8, work.data_ptr(),
                                    nbytes, torch.cuda.current_stream().cuda_stream)
        assert (work[nbytes:] == 0x55).all()
        assert not asked[0] or (out[0][:M, :K] == whole[0]).all()
        for t, (ref, bound), a in zip(out, refs, asked):
            n = ref.shape[0]
            assert ((t[:n, :K].double().cpu() - ref).abs() <= bound).all() if a else (t[:n, :K] == 7).all()
            assert (t[n:] == 7).all() and (t[:, K:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M,F,K", [(8, 6920, 5120), (17, 6920, 5120), (32, 2568, 16384), (32, 4000, 5120)])
def test_gradients_of_some_rows_in_long_walks(M, F, K):
    """Workgroups of 4 to 6 chunks of columns, the last of which ends inside a chunk (references in 64 bits on the device)."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen = torch.Generator(device=DEV).manual_seed(M)
    x, wg, wu, dh = (torch.randn(*s, generator=gen, device=DEV).mul_(scale).to(torch.bfloat16)
                     for s, scale in (((M, K), 1), ((F, K), 2 * K ** -0.5), ((F, K), K ** -0.5), ((M, F), 1)))
    _, saved = gated_linear_train(x, wg, wu)
    got = gated_linear_backward(dh, x, wg, wu, saved)
    for t, (ref, bound) in zip(got, _gated_grads(*(t.double() for t in (x, wg, wu, dh)), "silu")):
        assert ((t.double() - ref).abs() <= bound).all()


def test_codes_in_host_memory_reach_no_kernel(monkeypatch):
    """Weights and tokens in 8 bits that both lie in host memory (a checkpoint's, not yet moved) are refused, not handed on by their addresses."""
    from paper_2511_20426_amd import runner as R
    monkeypatch.setattr(B, "layer_linear_i8", lambda *a: pytest.fail("a host address went to the library"))
    monkeypatch.setattr(R, "_current_stream", lambda device: 0)
    x, w = (R.QuantizedRows.from_codes(torch.ones((n, 300), dtype=torch.int8), torch.ones(n)) for n in (4, 16))
    for out in (None, torch.empty((4, 16), dtype=torch.bfloat16)):
        with pytest.raises(AssertionError):
            R.linear_i8(x, w, out=out)
    with pytest.raises(AssertionError):
        R.linear_i8(torch.ones((4, 300), dtype=torch.bfloat16), w)


# factors of heads that lie beside each other in a wave: squares that fp32 holds, that pass its largest value, that it loses
SIZES = [1.0, 1e18, 1e20, 1e30, 1e37, 1e-18, 1e-22, 1e-30]


def _heads_of_all_sizes(gen, n, heads, D, t, sizes):
    x = torch.randn(n, 3, heads, D, generator=gen, dtype=torch.float64)
    return (x * torch.tensor(sizes, dtype=torch.float64)[torch.arange(n * 3 * heads) % len(sizes)].view(n, 3, heads, 1)).to(t).to(DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-6])
@pytest.mark.parametrize("dtype,D,heads", [("bf16", 128, 5), ("bf16", 128, 40), ("f32", 128, 3), ("f32", 64, 5), ("f32", 32, 11)])
def test_norms_of_values_whose_squares_leave_the_range(dtype, D, heads, eps):
    """Forward and on the way into the pool, over the whole range of the type."""
    grid, n, t = (1, 3), 9, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]      # (a block of the pool)
    pool, gen = _pool(heads, D, grid, dtype), _gen(heads)
    qkv, w = _heads_of_all_sizes(gen, n, heads, D, t, SIZES), [_normal(gen, D, dtype=t) for _ in range(2)]
    outs = pool.qk_norm_rope(qkv[:, 0], qkv[:, 1], w[0], w[1], 0, eps=eps)
    ang = _angles(D, grid, 0, n)
    for s in range(2):
        ref = _norm_rope(qkv[:, s].double().cpu(), w[s].double().cpu(), eps, ang)
        # (as test_norm_rope; bringing a head into the range is exact)
        assert ((outs[s].double().cpu() - ref).abs() <= ref.abs() * HALF[t] + _pairs(ref) * 2 * WAY + 1e-30).all()
    pool.append_batch([0], [0], 0, [qkv[:, 1]], [qkv[:, 2]], k_weight=w[1], eps=eps)
    per = 2 * 128 * D
    for h in range(heads):
        at = pool.ctx.kv_cache_page_index(0, 0, h)
        k = pool.pool[at * per * t.itemsize:(at + 1) * per * t.itemsize].view(t).view(2, 128, D)[0]
        if dtype == "bf16":
            c = torch.arange(16, device=DEV)[None] ^ (torch.arange(128, device=DEV)[:, None] & 15)
            k = k.view(128, 16, 8).gather(1, c[:, :, None].expand(128, 16, 8)).view(128, D)
        assert (k[:n] == outs[1][:, h]).all() and (k[n:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("dtype,D,heads,n", [("bf16", 128, 5, 9), ("bf16", 128, 40, 3), ("f32", 64, 5, 70), ("f32", 32, 11, 5)])
def test_gradients_of_norms_whose_squares_leave_the_range(dtype, D, heads, n, eps):
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    pool, gen = _pool(heads, D, (4, 5), dtype), _gen(n + 1)
    qkv = _heads_of_all_sizes(gen, n, heads, D, t, [1.0, 1e18, 1e20, 1e25, 1e-18, 1e-22])
    dz, w = _normal(gen, n, heads, 2, D, dtype=t), [_normal(gen, D, dtype=t) for _ in range(2)]
    got = pool.qk_norm_rope_backward(dz[:, :, 0], dz[:, :, 1], qkv[:, 0], qkv[:, 1], w[0], w[1], 2, eps=eps)
    ang = _angles(D, (4, 5), 2, n)
    for s in range(2):
        dx, dw, size, size_w = _norm_grads(dz[:, :, s].double().cpu(), qkv[:, s].double().cpu(), w[s].double().cpu(), eps, ang)
        # (as test_norm_rope_backward)
        assert ((got[s].double().cpu() - dx).abs() <= dx.abs() * HALF[t] + size * 3 * WAY + 1e-38).all()
        assert ((got[2 + s].double().cpu() - dw).abs() <= size_w * (2 * WAY + 128 * 2.0 ** -24) + 1e-30).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 32)])
def test_heads_that_are_not_finite(dtype, D):
    """... stay by themselves: the heads beside them in the wave have the bits that they have without them."""
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    pool, gen = _pool(9, D, (4, 5), dtype), _gen(4)
    x, w = _normal(gen, 6, 9, D, dtype=t), _normal(gen, D, dtype=t)
    fine = pool.qk_norm_rope(x, None, w, None, 0)[0]
    x[1, 2, 5], x[3, 4, 7], x[5, 8, 0] = float("inf"), float("nan"), -float("inf")
    y = pool.qk_norm_rope(x, None, w, None, 0)[0]
    bad = torch.zeros((6, 9), dtype=torch.bool, device=DEV)
    bad[1, 2] = bad[3, 4] = bad[5, 8] = True
    assert (y[~bad] == fine[~bad]).all() and y[bad].isnan().any(-1).all()


@pytest.mark.parametrize("rows", [1, 2, 16, 32])
def test_few_tokens_of_too_many_columns_are_refused(rows):
    """Their launch would have 2^32 threads."""
    n, p = (1 << 28) - 8, 4096
    for call in (lambda: B.layer_linear_i8(p, p, p, p, p, rows, n, 200, 256, 256, n),
                 lambda: B.layer_linear_i8_values(p, B.CA_BF16, p, p, p, rows, n, 200, 200, 256, n, p, 1 << 30),
                 lambda: B.layer_gated_bf16(p, p, p, p, 0, B.CA_SILU, rows, n, 128, 128, 128, 128, n)):
        with pytest.raises(B.CascadeAttnError) as e:
            call()
        assert e.value.code == B.CA_EUNSUPPORTED


@pytest.mark.parametrize("mt", [4, 6])
def test_where_the_projections_of_many_columns_lie(mt):
    """A row of blocks of 2^32 bytes: the generated program followed over a tile of several such rows, at the last columns."""
    from tests import test_gemm_op_rows as T
    N = (1 << 26) + 40
    T.test_loop_over_tiles("gated", True, mt, (32 * mt + 20, N, 256), [(0, N // 128), (1, N // 128 - 1)], 0, 10)
