"""Layer norm with weights of groups of rows, and its gradients, against plain implementations in 64 bits, against differences, and its refusals."""
import pytest
import torch

from paper_2511_20426_amd import binding as B

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}        # a rounding, relative: half a step
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "f32": torch.float32}
# A thread adds 8 values of up to six pieces, six exchanges join a wave and up to 16 additions its row: a chain of at most 48 + 6 + 4 fp32
# roundings (four waves of six pieces; sixteen have up to four: 32 + 6 + 16) of the sum of magnitudes, in the mean and in the squares (of which the root halves the error); products, root and quotient
# are some ten more.
WAY = 72 * 2.0 ** -24


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _normal(gen, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(dtype).to(DEV)


def _plain(x, w, b, eps):
    """y, n, r, and how far fp32 may be off in n: the mean, held in fp32, is off by a rounding of itself and, corrected, by what is left
    of the sum's; differences and r by WAY"""
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    r = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    off = r * (2.0 ** -23 * mean.abs() + WAY * d.abs().mean(-1, keepdim=True)) + 2 * WAY * (d * r).abs()
    return d * r * w + b, d * r, r, off


def _by_row(t, rows, width):
    return t.double().cpu().reshape(-1, width).repeat_interleave(rows // (t.numel() // width), 0)


# rows, width, groups, type, the weights' type: single values and rows, odd widths, the borders of a wave's, four waves' and sixteen waves' rows
NORMS = [(1, 1, 1, "bf16", "f32"), (3, 5, 1, "f32", "f32"), (1, 5120, 1, "bf16", "bf16"), (9, 8, 3, "bf16", "f32"), (433, 129, 1, "f32", "f32"),
         (6, 2048, 3, "bf16", "f32"), (7, 2047, 7, "bf16", "bf16"), (10, 2056, 5, "f32", "f32"), (5, 8192, 1, "bf16", "f32"), (4, 8193, 2, "bf16", "f32"),
         (3, 32768, 1, "f32", "f32"), (2, 30001, 1, "bf16", "bf16"), (1205, 1536, 5, "bf16", "f32"), (600, 4096, 2, "bf16", "f32"), (70, 520, 1, "bf16", "bf16"),
         (12, 2560, 3, "bf16", "f32"), (7, 2561, 1, "f32", "f32"), (9, 2553, 1, "f32", "f32"), (6, 10240, 2, "bf16", "bf16"), (5, 10233, 1, "f32", "f32"),
         (5, 12288, 1, "bf16", "f32"), (6, 12281, 1, "f32", "f32"), (4, 12289, 2, "bf16", "bf16"), (5, 16384, 1, "f32", "f32"),
         # as many rows as are dealt to two and three workgroups on a CU, and groups that they do not come out even for
         (4705, 264, 5, "bf16", "f32"), (6150, 2568, 3, "bf16", "bf16"), (4100, 2568, 1, "f32", "f32"), (1030, 8, 515, "bf16", "f32")]


def _case(rows, width, groups, dtype, w_dtype):
    gen = _gen(rows * 7 + width)
    x = _normal(gen, rows, width, scale=2.0) + _normal(gen, width)
    x[0] = 0
    if rows > 2:
        x[1] = 3.5                                                   # equal values
        x[2] = x[2] * 1e-3 + 100                                     # far from zero
    if rows > 4:
        x[3] *= 1e-18
        x[4] = 0
        x[4, width // 2] = 1000
    shape = (groups, width) if groups > 1 else (width,)
    return x.to(T[dtype]), _normal(gen, *shape, dtype=T[w_dtype]), _normal(gen, *shape, dtype=T[w_dtype]), _normal(gen, rows, width, dtype=T[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["both", "weight", "bias", "none"])
@pytest.mark.parametrize("rows,width,groups,dtype,w_dtype", NORMS)
def test_forward(rows, width, groups, dtype, w_dtype, which):
    from paper_2511_20426_amd.runner import layer_norm
    x, weight, bias, _ = _case(rows, width, groups, dtype, w_dtype)
    keep = x.clone()
    y = layer_norm(x, weight if which in ("both", "weight") else None, bias if which in ("both", "bias") else None)
    assert y.dtype == x.dtype and torch.equal(x, keep)
    w = _by_row(weight, rows, width) if which in ("both", "weight") else torch.ones(rows, width, dtype=torch.float64)
    b = _by_row(bias, rows, width) if which in ("both", "bias") else torch.zeros(rows, width, dtype=torch.float64)
    ref, _, _, off = _plain(x.double().cpu(), w, b, 1e-6)
    assert ((y.double().cpu() - ref).abs() <= HALF[y.dtype] * 1.01 * ref.abs() + w.abs() * off + 1e-37).all()


def _grads(dy, x, w, eps):
    _, n, r, off = _plain(x, w, 0 * w, eps)
    dn = dy * w
    mean, dot = dn.mean(-1, keepdim=True), (dn * n).mean(-1, keepdim=True)
    dx = r * (dn - mean - n * dot)
    # sums as above; n's error in the product with the dot, and in the dot
    bound = r * (WAY * (dn.abs() + dn.abs().mean(-1, keepdim=True) + n.abs() * (dn * n).abs().mean(-1, keepdim=True)) + off * dot.abs() +
                 n.abs() * (dn.abs() * off).mean(-1, keepdim=True)) + 2 * WAY * dx.abs()
    return dx, bound, dy * n, dy.abs() * off


@pytest.mark.gpu
@pytest.mark.parametrize("rows,width,groups,dtype,w_dtype", NORMS)
def test_gradients(rows, width, groups, dtype, w_dtype):
    from paper_2511_20426_amd.runner import layer_norm_backward
    x, weight, bias, dy = _case(rows, width, groups, dtype, w_dtype)
    dx, dw, db = layer_norm_backward(dy, x, weight, bias)
    ref, bound, dwr, dwo = _grads(dy.double().cpu(), x.double().cpu(), _by_row(weight, rows, width), 1e-6)
    assert dx.dtype == x.dtype and ((dx.double().cpu() - ref).abs() <= HALF[dx.dtype] * 1.01 * ref.abs() + bound + 1e-37).all()
    assert dw.shape == weight.shape and db.shape == bias.shape and dw.dtype == db.dtype == torch.float32
    # a thread's rows (at most the group's), four waves' and one rounding
    CHAIN = (rows // groups + 6) * 2.0 ** -24
    each = lambda t: t.reshape(groups, -1, width).sum(1)             # noqa: E731
    dyd = dy.double().cpu()
    for got, terms, more in ((dw, dwr, dwo), (db, dyd, 0 * dyd)):
        want = each(terms)
        assert ((got.double().cpu().reshape(groups, width) - want).abs() <= each(more) + CHAIN * each(terms.abs()) + 1e-37).all()
    # each gradient by itself, and none
    dx1, dw1, none = layer_norm_backward(dy, x, weight, None)
    assert none is None and torch.equal(dx1, dx) and torch.equal(dw1, dw)
    ones = torch.ones_like(weight)
    dx2, dw2, db2 = layer_norm_backward(dy, x, None, bias)
    assert dw2 is None and torch.equal(db2, db) and torch.equal(dx2, layer_norm_backward(dy, x, ones)[0])
    dx3 = layer_norm_backward(dy, x)
    assert dx3[1] is None and dx3[2] is None and torch.equal(dx3[0], dx2)


@pytest.mark.gpu
@pytest.mark.parametrize("groups", [1, 2])
def test_gradients_against_differences(groups):
    """The loss sum(c y) in 64 bits, from the plain form at x +- h: the quotient is off by h^2 and by roundings of 2^-52 / h"""
    from paper_2511_20426_amd.runner import layer_norm_backward
    gen, rows, width, h = _gen(5), 4, 11, 1e-5
    x, c = _normal(gen, rows, width), _normal(gen, rows, width)
    w, b = _normal(gen, groups, width), _normal(gen, groups, width)
    if groups == 1:
        w, b = w[0], b[0]
    got = layer_norm_backward(c, x, w, b)
    xd, wd, bd, cd = (t.double().cpu() for t in (x, w, b, c))

    def loss(xd, wd, bd):
        each = lambda t: t.reshape(-1, width).repeat_interleave(rows // groups, 0)      # noqa: E731
        return (cd * _plain(xd, each(wd), each(bd), 1e-6)[0]).sum()

    for k, g in enumerate(got):
        args = [xd, wd, bd]
        for i in range(g.numel()):
            step = torch.zeros(g.numel(), dtype=torch.float64)
            step[i] = h
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + step.view(args[k].shape), args[k] - step.view(args[k].shape)
            assert abs((loss(*up) - loss(*down)) / (2 * h) - g.flatten()[i].item()) < 2e-5 * (1 + abs(g.flatten()[i].item()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("width", [96, 97, 2600, 9000])
def test_strides_alignment_in_place_and_streams(dtype, width):
    """Columns of a wider tensor from an odd place on, results into one and over the inputs, on another stream: the bits of packed tensors, and nothing
    beside them."""
    from paper_2511_20426_amd.runner import layer_norm, layer_norm_backward
    gen, rows, t = _gen(width), 12, T[dtype]
    wide, wide_dy = _normal(gen, rows, 2 * width + 11, dtype=t), _normal(gen, rows, width + 5, dtype=t)
    w, b = _normal(gen, 2, 4 * width + 1)[:, 1:width + 1], _normal(gen, 2, 4 * width + 1)[:, 1:width + 1]
    x, dy = wide[:, 3:3 + width], wide_dy[:, 5:]
    # (packed rows may be added in another order: they are loaded in another)
    ref = layer_norm(x, w, b)
    dref = layer_norm_backward(dy, x, w, b)
    xd, wd, bd = x.double().cpu(), _by_row(w.contiguous(), rows, width), _by_row(b.contiguous(), rows, width)
    plain, _, _, off = _plain(xd, wd, bd, 1e-6)
    assert ((ref.double().cpu() - plain).abs() <= HALF[t] * 1.01 * plain.abs() + wd.abs() * off).all()
    out = torch.full((rows, width + 9), 7.0, dtype=t, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer_norm(x, w, b, out=out[:, 4:4 + width])
        got = layer_norm_backward(dy, x, w, b, dx=dy)
        layer_norm(x, w, b, out=x)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out[:, 4:4 + width], ref) and (out[:, :4] == 7).all() and (out[:, 4 + width:] == 7).all()
    assert torch.equal(x, ref) and all(torch.equal(p, q) for p, q in zip(got, dref)) and got[0] is dy


@pytest.mark.gpu
@pytest.mark.parametrize("width", [40, 43, 3000])
def test_values_beyond_the_squares_of_fp32(width):
    """Rows of 1e30 and 1e-25 (with an eps of their own size), a row whose sum leaves fp32, infinities and NaN."""
    from paper_2511_20426_amd.runner import layer_norm, layer_norm_backward
    gen = _gen(width)
    x = _normal(gen, 6, width)
    x[0] *= 1e30
    x[1] = 3e38 * (1 - 0.2 * torch.rand(width, generator=gen).to(DEV))
    x[2] *= 1e-25
    x[3] = 1e20
    x[4, 3] = float("inf")
    x[5, 1] = float("nan")
    dy, one = _normal(gen, 6, width), torch.ones(1, width, dtype=torch.float64)
    for eps in (1e-6, 1e-52, 0.0):
        eps = float(torch.tensor(eps, dtype=torch.float32))          # 1e-52 is zero in fp32
        y = layer_norm(x, eps=eps).double().cpu()
        dx = layer_norm_backward(dy, x, eps=eps)[0].double().cpu()
        for i in (0, 1, 2):
            ref, _, _, off = _plain(x[i:i + 1].double().cpu(), one, 0 * one, eps)
            assert ((y[i] - ref[0]).abs() <= 2.0 ** -24 * ref[0].abs() + off[0] + 1e-37).all(), (eps, i)
            ref, bound, _, _ = _grads(dy[i:i + 1].double().cpu(), x[i:i + 1].double().cpu(), one, eps)
            ok = (dx[i] - ref[0]).abs() <= 2.0 ** -24 * ref[0].abs() + bound[0] + 2.0 ** -146        # (results below the normal numbers: steps of 2^-149)
            assert ok.all(), (eps, i)
        assert (y[3] == 0).all() if eps else y[3].isnan().all()
        assert y[4].isnan().all() and y[5].isnan().all()


@pytest.mark.gpu
def test_no_rows():
    from paper_2511_20426_amd.runner import layer_norm, layer_norm_backward
    for shape in ((40,), (3, 40)):
        w = torch.ones(shape, device=DEV)
        x = torch.empty((0, 40), device=DEV)
        assert layer_norm(x, w, w).shape == (0, 40)
        dx, dw, db = layer_norm_backward(x, x, w, w)
        assert dx.shape == (0, 40) and dw.shape == shape and (dw == 0).all() and (db == 0).all()


@pytest.mark.gpu
def test_same_bits_every_time_and_in_replayed_graphs():
    """Two captured graphs of calls with workspaces, replayed in turn with eager work between them."""
    from paper_2511_20426_amd.runner import layer_norm, layer_norm_backward
    gen = _gen(1)
    sets = []
    for rows, width in ((900, 640), (301, 5120)):
        x, dy = _normal(gen, rows, width, dtype=torch.bfloat16), _normal(gen, rows, width, dtype=torch.bfloat16)
        sets.append((x, dy, _normal(gen, width), _normal(gen, width)))

    def run(x, dy, w, b):
        return (layer_norm(x, w, b),) + layer_norm_backward(dy, x, w, b)

    eager = [run(*s) for s in sets]
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(*s))
        graphs.append(g)
    for trip in range(3):
        for t in outs[0] + outs[1]:
            t.zero_()
        for g in graphs:
            g.replay()
        again = [run(*s) for s in sets]
        torch.cuda.synchronize()
        for want, got, more in zip(eager, outs, again):
            assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(want, got, more)), trip
    # another x in place, the same graph
    sets[0][0].copy_(_normal(gen, 900, 640))
    graphs[0].replay()
    assert all(torch.equal(p, q) for p, q in zip(run(*sets[0]), outs[0]))


@pytest.mark.gpu
def test_arguments_refused_on_device():
    from paper_2511_20426_amd.runner import layer_norm, layer_norm_backward
    x, w = torch.zeros((6, 16), device=DEV), torch.ones(16, device=DEV)
    for bad in (lambda: layer_norm(x.half()), lambda: layer_norm(x[0]), lambda: layer_norm(x, w[:8]), lambda: layer_norm(x, w.bfloat16()),
                lambda: layer_norm(x, w.expand(4, 16).contiguous()), lambda: layer_norm(x, w, w.bfloat16()), lambda: layer_norm(x.t()),
                lambda: layer_norm(x, w, out=x.bfloat16()), lambda: layer_norm(x, w, out=x[:3]), lambda: layer_norm(x, w.cpu()),
                lambda: layer_norm_backward(x[:5], x, w), lambda: layer_norm_backward(x.bfloat16(), x, w)):
        with pytest.raises(AssertionError):
            bad()
    for bad in (lambda: layer_norm(x, w, eps=-1.0), lambda: layer_norm(x, w, eps=float("nan")), lambda: layer_norm(x[:1].expand(6, 16), w)):
        with pytest.raises(B.CascadeAttnError):
            bad()


def test_arguments_refused():
    """On the host, before anything is launched"""
    p = 4096
    good = dict(x=p, dtype=B.CA_BF16, w=p, b=p, w_dtype=B.CA_F32, eps=1e-6, y=p, rows=6, width=64, groups=2, ldx=64, ldw=64, ldy=64)
    for change, code in ((dict(rows=-1), B.CA_EINVAL), (dict(groups=0), B.CA_EINVAL), (dict(groups=4), B.CA_EINVAL), (dict(eps=-1.0), B.CA_EINVAL),
                         (dict(eps=float("inf")), B.CA_EINVAL), (dict(dtype=7), B.CA_EINVAL), (dict(w_dtype=-1), B.CA_EINVAL),
                         (dict(dtype=B.CA_F32, w_dtype=B.CA_BF16), B.CA_EINVAL), (dict(x=0), B.CA_EINVAL), (dict(y=0), B.CA_EINVAL),
                         (dict(x=p + 1), B.CA_EINVAL), (dict(y=p + 1), B.CA_EINVAL), (dict(w=p + 2), B.CA_EINVAL), (dict(b=p + 1), B.CA_EINVAL),
                         (dict(ldx=63), B.CA_EINVAL), (dict(ldy=0), B.CA_EINVAL), (dict(ldw=63), B.CA_EINVAL), (dict(width=0), B.CA_EUNSUPPORTED),
                         (dict(width=32769, ldx=32769, ldy=32769, ldw=32769), B.CA_EUNSUPPORTED), (dict(rows=2 ** 30 + 2), B.CA_EUNSUPPORTED),
                         (dict(rows=2 ** 21, groups=2 ** 21), B.CA_EUNSUPPORTED)):
        with pytest.raises(B.CascadeAttnError) as e:
            B.layer_norm(*{**good, **change}.values())
        assert e.value.code == code, change
    B.layer_norm(*{**good, "rows": 0, "x": 0, "y": 0}.values())
    back = dict(dy=p, x=p, dtype=B.CA_BF16, w=p, w_dtype=B.CA_F32, eps=1e-6, dx=p, dw=p, db=p, rows=600, width=64, groups=2, lddy=64, ldx=64, ldw=64, lddx=64,
                work=p, nbytes=1 << 30)
    need = B.layer_norm_backward_workspace(600, 64, 2)
    assert need > 0 and B.layer_norm_backward_workspace(600, 64, 7) == 0 and B.layer_norm_backward_workspace(-2, 64, 2) == 0
    for change in (dict(dy=0), dict(dx=0), dict(x=0), dict(dw=p + 2), dict(db=p + 1), dict(lddy=63), dict(lddx=63), dict(work=0), dict(work=p + 8),
                   dict(nbytes=need - 1), dict(rows=601)):
        with pytest.raises(B.CascadeAttnError) as e:
            B.layer_norm_backward(*{**back, **change}.values())
        assert e.value.code == B.CA_EINVAL, change
