"""The linear map with low-rank adapters of many requests, and its gradients, against plain implementations in 64 bits, against differences, and refusals."""
import pytest
import torch

from paper_2511_20426_amd import binding as B

HALF = 2.0 ** -8                                                     # a rounding to bf16, relative: half a step
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _normal(gen, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(torch.bfloat16).to(DEV)


def _index(gen, m, g, how):
    """which adapter each row has"""
    if how == "mixed":                                               # numbers that are no adapter's among them
        index = torch.randint(-1, g + 1, (m,), generator=gen)
        index[::7] = torch.tensor([-2 ** 31, 2 ** 31 - 1, -1, g])[torch.randint(0, 4, (len(index[::7]),), generator=gen)]
    elif how == "runs":
        index = torch.arange(m) * g // m
    else:
        index = torch.full((m,), -1)
    return index.to(torch.int32).to(DEV)


def _case(m, n, k, g, r, how):
    gen = _gen(m * 3 + n + r)
    return (_normal(gen, m, k), _normal(gen, n, k, scale=k ** -0.5), _normal(gen, g, r, k, scale=k ** -0.5), _normal(gen, g, n, r, scale=r ** -0.5),
            (0.5 + torch.rand(g, generator=gen)).to(DEV), _index(gen, m, g, how), _normal(gen, m, n))


def _adapted(x, w, down, up, scales, index):
    """y, T, and how far bf16 operands with fp32 sums may be off.  A value of T is rounded once to bf16, behind a sum of k products in fp32; y's sums are of k and
    of r products, an order of any kind being off by less than a rounding of 2^-24 of all magnitudes for each."""
    x, w, down, up, scales = (t.double().cpu() for t in (x, w, down, up, scales))
    (m, k), r = x.shape, down.shape[1]
    y, t = x @ w.T, torch.zeros(m, r, dtype=torch.float64)
    off = k * 2.0 ** -24 * (x.abs() @ w.abs().T)
    for g in range(down.shape[0]):
        of = index.cpu() == g
        t[of] = scales[g] * (x[of] @ down[g].T)
        y[of] += t[of] @ up[g].T
        t_off = HALF * t[of].abs() + 1.01 * (k + 2) * 2.0 ** -24 * scales[g] * (x[of].abs() @ down[g].abs().T)
        off[of] += 1.01 * t_off @ up[g].abs().T + (r + 2) * 2.0 ** -24 * (t[of].abs() @ up[g].abs().T)
    return y, t, off


def _close(got, ref, off):
    err = (got.double().cpu() - ref).abs()
    assert (err <= 1.01 * HALF * ref.abs() + 1.01 * off + 1e-37).all(), (err - HALF * ref.abs() - off).max()


# rows, columns, k, adapters, rank, which rows have which: single tokens, the borders of the kernels for few and many rows, odd sizes and ranks
CASES = [(16, 5120, 256, 3, 16, "mixed"), (16, 5128, 128, 3, 16, "mixed"), (3, 27312, 128, 2, 32, "mixed"), (31, 2648, 256, 4, 64, "mixed"), (40, 384, 2048, 3, 16, "mixed"),
         (512, 136, 4224, 2, 100, "mixed"), (513, 128, 2176, 2, 32, "runs"), (33, 128, 13824, 5, 64, "mixed"),
         (1, 8, 128, 1, 1, "runs"), (2, 24, 5120, 3, 32, "mixed"), (32, 40, 1152, 7, 128, "mixed"), (20, 56, 4096, 2, 64, "none"), (40, 8, 256, 2, 4, "mixed"), (1, 776, 1024, 8, 16, "mixed"), (5, 1032, 384, 3, 5, "mixed"), (16, 264, 640, 5, 40, "mixed"), (17, 264, 256, 4, 128, "mixed"),
         (32, 136, 256, 32, 64, "mixed"), (32, 136, 256, 2, 8, "none"), (33, 136, 256, 3, 33, "mixed"), (257, 776, 1024, 6, 5, "mixed"), (600, 520, 256, 5, 100, "runs"),
         (300, 1536, 1536, 1, 32, "runs"), (1205, 1288, 512, 7, 64, "mixed"), (260, 512, 384, 2, 64, "none"), (2100, 2560, 256, 3, 128, "runs"),
         (8195, 264, 128, 3, 20, "mixed"), (8210, 136, 256, 2, 64, "runs"), (8300, 128, 256, 4, 128, "mixed")]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,g,r,how", CASES)
def test_forward(m, n, k, g, r, how):
    from paper_2511_20426_amd.runner import Adapters, linear_adapted, linear_adapted_train
    x, w, down, up, scales, index, _ = _case(m, n, k, g, r, how)
    keep = [t.clone() for t in (x, w, down, up, index)]
    adapters = Adapters.from_weights(down, up, scales)
    y, saved = linear_adapted_train(x, w, adapters, index)
    assert all(torch.equal(a, b) for a, b in zip(keep, (x, w, down, up, index)))
    ref, t, off = _adapted(x, w, down, up, scales, index)
    _close(y, ref, off)
    way = 1.01 * (k + 2) * 2.0 ** -24 * 1.5 * (x.double().cpu().abs() @ down.double().cpu().abs().amax(0).T)
    _close(saved[0, :, :r], t, way)
    # ... and what the rounding left: a half step of a half step is between their sum and T
    assert ((saved[:, :, :r].double().cpu().sum(0) - t).abs() <= 1.01 * HALF * HALF * t.abs() + 1.01 * way).all()
    none = (index.cpu() < 0) | (index.cpu() >= g)
    assert (saved[:, :, r:] == 0).all() and (saved.cpu()[:, none] == 0).all()
    assert torch.equal(linear_adapted(x, w, adapters, index), y)


# ... whose columns are whole steps of 128
GRADS = [c for c in CASES if c[1] % 128 == 0] + [(1, 128, 128, 2, 3, "mixed"), (7, 384, 256, 3, 32, "mixed"), (33, 256, 128, 40, 64, "mixed"), (700, 640, 384, 5, 100, "mixed"),
                                                 (64, 128, 128, 1, 1, "runs"), (4100, 128, 128, 1, 128, "runs"), (1000, 256, 1152, 2, 33, "runs")]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,g,r,how", GRADS)
def test_gradients(m, n, k, g, r, how):
    from paper_2511_20426_amd.runner import Adapters, linear_adapted_backward, linear_adapted_train
    x, w, down, up, scales, index, dy = _case(m, n, k, g, r, how)
    adapters = Adapters.from_weights(down, up, scales)
    _, saved = linear_adapted_train(x, w, adapters, index)
    got = linear_adapted_backward(dy, x, w.t().contiguous(), adapters, index, saved)
    assert got[0].shape == (m, k) and got[1].shape == (g, r, k) and got[2].shape == (g, n, r) and all(t.dtype == torch.bfloat16 and t.is_contiguous() for t in got)
    # dx: the same map with the transposed matrices
    dx, u, off = _adapted(dy, w.t(), up.transpose(1, 2), down.transpose(1, 2), scales, index)
    _close(got[0], dx, off)
    t = _adapted(x, w, down, up, scales, index)[1]
    xd, dyd = x.double().cpu(), dy.double().cpu()
    for a in range(g):
        of = index.cpu() == a
        # the operand of the rank is rounded to bf16 twice, behind a sum in fp32; the sum over the rows, in fp32 too, is joined from up to 64 parts
        for low, wide, mine, of_sum in ((u, xd, got[1][a], k), (t, dyd, got[2][a].t(), n)):
            _close(mine, low[of].T @ wide[of], ((HALF * HALF + (2 * of.sum() + 70) * 2.0 ** -24) * low[of].abs() + 2.0 ** -24 * 4096 * low[of].abs().mean()).T @ wide[of].abs()
                   if of.any() else torch.zeros(mine.shape, dtype=torch.float64))
    none, d_down, d_up = linear_adapted_backward(dy, x, None, adapters, index, saved)
    assert none is None and torch.equal(d_down, got[1]) and torch.equal(d_up, got[2])


@pytest.mark.gpu
def test_gradients_against_differences():
    """The loss sum(c y) in 64 bits is linear in each argument: its difference over a step of 1 is its derivative, but for roundings"""
    from paper_2511_20426_amd.runner import Adapters, linear_adapted_backward, linear_adapted_train
    m, n, k, g, r = 6, 128, 128, 2, 2
    x, w, down, up, scales, index, c = _case(m, n, k, g, r, "mixed")
    index = torch.tensor([0, 1, -1, 1, 0, 5], dtype=torch.int32, device=DEV)
    adapters = Adapters.from_weights(down, up, scales)
    _, saved = linear_adapted_train(x, w, adapters, index)
    got = linear_adapted_backward(c, x, w.t().contiguous(), adapters, index, saved)
    args = [x.double(), down.double(), up.double()]

    def loss(x, down, up):
        return (c.double().cpu() * _adapted(x, w, down, up, scales, index)[0]).sum().item()

    gen, zero = _gen(0), loss(*args)
    for which, grad in enumerate(got):
        size = grad.double().norm().item() / grad.numel() ** 0.5
        for at in torch.randint(0, grad.numel(), (25,), generator=gen).tolist():
            moved = [t.clone() for t in args]
            moved[which].view(-1)[at] += 1
            assert abs(loss(*moved) - zero - grad.flatten()[at].item()) <= 0.02 * size + HALF * abs(grad.flatten()[at].item())


@pytest.mark.gpu
@pytest.mark.parametrize("m", [9, 32, 130, 700])
def test_no_request_touches_another(m):
    """Infinities and NaN in one adapter, in its scale, and in rows: the others' bits stay"""
    from paper_2511_20426_amd.runner import Adapters, linear_adapted_backward, linear_adapted_train
    n, k, g, r = 256, 256, 4, 32
    x, w, down, up, scales, index, dy = _case(m, n, k, g, r, "mixed")
    index[1:4] = torch.tensor([0, 2, -1], dtype=torch.int32)
    w_t = w.t().contiguous()
    adapters = Adapters.from_weights(down, up, scales)
    y, saved = linear_adapted_train(x, w, adapters, index)
    grads = linear_adapted_backward(dy, x, w_t, adapters, index, saved)
    for bad in (float("inf"), float("nan")):
        down2, up2, scales2, x2, dy2 = down.clone(), up.clone(), scales.clone(), x.clone(), dy.clone()
        down2[2, 3, 5], up2[2, 7], scales2[2], x2[2, 0], dy2[2, 0] = bad, bad, bad, bad, bad
        poisoned = Adapters.from_weights(down2, up2, scales2)
        other = index != 2
        other[2] = False
        y2, saved2 = linear_adapted_train(x2, w, poisoned, index)
        assert torch.equal(y2[other], y[other]) and torch.equal(saved2[:, other], saved[:, other]) and not y2[2].isfinite().any()
        dx, d_down, d_up = linear_adapted_backward(dy2, x2, w_t, poisoned, index, saved2)
        keep = [0, 1, 3]
        assert torch.equal(dx[other], grads[0][other]) and torch.equal(d_down[keep], grads[1][keep]) and torch.equal(d_up[keep], grads[2][keep])


@pytest.mark.gpu
@pytest.mark.parametrize("m", [1, 20, 300])
def test_strides_and_streams(m):
    """Columns of wider tensors, results into one, on another stream: the bits of packed tensors, and nothing beside them"""
    from paper_2511_20426_amd.runner import Adapters, linear_adapted, linear_adapted_backward, linear_adapted_train
    n, k, g, r = 384, 256, 3, 24
    x, w, down, up, scales, index, dy = _case(m, n, k, g, r, "mixed")
    adapters, w_t = Adapters.from_weights(down, up, scales), w.t().contiguous()
    y, saved = linear_adapted_train(x, w, adapters, index)
    ref = linear_adapted_backward(dy, x, w_t, adapters, index, saved)

    def wide(t, before, behind):
        room = torch.full((t.shape[0], before + t.shape[1] + behind), 7.0, dtype=t.dtype, device=DEV)
        room[:, before:before + t.shape[1]] = t
        return room, room[:, before:before + t.shape[1]]

    xs, ws, dys, wts = (wide(t, 8, 16)[1] for t in (x, w, dy, w_t))
    room, out = wide(torch.zeros_like(y), 16, 24)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        assert linear_adapted(xs, ws, adapters, index, out=out) is out
        got = linear_adapted_backward(dys, xs, wts, adapters, index, saved)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, y) and (room[:, :16] == 7).all() and (room[:, 16 + n:] == 7).all()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))


@pytest.mark.gpu
def test_no_rows():
    from paper_2511_20426_amd.runner import Adapters, linear_adapted_backward, linear_adapted_train
    x, w, down, up, scales, index, dy = _case(3, 256, 128, 2, 8, "mixed")
    adapters = Adapters.from_weights(down, up, scales)
    y, saved = linear_adapted_train(x[:0], w, adapters, index[:0])
    assert y.shape == (0, 256)
    dx, d_down, d_up = linear_adapted_backward(dy[:0], x[:0], w.t().contiguous(), adapters, index[:0], saved)
    assert dx.shape == (0, 128) and (d_down == 0).all() and (d_up == 0).all()


@pytest.mark.gpu
def test_same_bits_every_time_and_in_replayed_graphs():
    """Graphs of calls with workspaces, replayed in turn, with other rows and other adapters of the rows in the same tensors"""
    from paper_2511_20426_amd.runner import Adapters, linear_adapted_backward, linear_adapted_train
    sets = []
    for m, n, k, g, r in ((700, 640, 384, 5, 32), (6, 384, 256, 3, 16)):
        x, w, down, up, scales, index, dy = _case(m, n, k, g, r, "mixed")
        sets.append((x, w, Adapters.from_weights(down, up, scales), index, dy, w.t().contiguous()))

    def run(x, w, adapters, index, dy, w_t):
        y, saved = linear_adapted_train(x, w, adapters, index)
        return (y,) + linear_adapted_backward(dy, x, w_t, adapters, index, saved)

    for s in sets:
        run(*s)
    graphs, outs = [], []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(run(*s))
        graphs.append(graph)
    gen = _gen(8)
    for trip in range(3):
        for x, _, adapters, index, _, _ in sets:
            x.copy_(torch.randn(x.shape, generator=gen))
            index.copy_(_index(gen, len(index), adapters.down.shape[0], ("mixed", "runs", "none")[trip]))
        for graph in graphs:
            graph.replay()
        for s, out in zip(sets, outs):
            again = run(*s)
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(again, out)), trip


@pytest.mark.gpu
def test_weights_in_place_and_filled_up():
    from paper_2511_20426_amd.runner import Adapters
    down, up = _normal(_gen(0), 2, 32, 128), _normal(_gen(1), 2, 8, 32)
    a = Adapters.from_weights(down, up)
    assert a.down.data_ptr() == down.data_ptr() and a.up.data_ptr() == up.data_ptr() and a.scales.tolist() == [1, 1] and a.rank == 32
    for r, room in ((1, 32), (33, 64), (65, 128)):
        down, up = _normal(_gen(0), 2, r, 128).float(), _normal(_gen(1), 2, 8, r).float()
        a = Adapters.from_weights(down, up, torch.tensor([2.0, 3.0], dtype=torch.float64, device=DEV))
        assert a.down.shape == (2, room, 128) and a.up.shape == (2, 8, room) and a.rank == r and a.scales.dtype == torch.float32
        assert torch.equal(a.down[:, :r].float(), down) and torch.equal(a.up[:, :, :r].float(), up) and (a.down[:, r:] == 0).all() and (a.up[:, :, r:] == 0).all()


@pytest.mark.gpu
def test_arguments_refused_on_device():
    from paper_2511_20426_amd.runner import Adapters, linear_adapted, linear_adapted_backward, linear_adapted_train
    x, w, down, up, scales, index, dy = _case(40, 256, 128, 2, 8, "mixed")
    a = Adapters.from_weights(down, up, scales)
    y, saved = linear_adapted_train(x, w, a, index)
    w_t = w.t().contiguous()
    for bad in (lambda: linear_adapted(x, w, a, index.long()), lambda: linear_adapted(x, w, a, index[:39]), lambda: linear_adapted(x, w, a, index.cpu()),
                lambda: linear_adapted(x.float(), w, a, index), lambda: linear_adapted(x, w[:248], a, index), lambda: linear_adapted(x[:, :64], w[:, :64], a, index),
                lambda: linear_adapted(x, w, a, index, out=y.float()), lambda: linear_adapted(x, w.t(), a, index), lambda: linear_adapted(x, w, a, index[::2]),
                lambda: Adapters.from_weights(_normal(_gen(0), 1, 129, 128), _normal(_gen(0), 1, 8, 129)), lambda: Adapters.from_weights(down, up[:1]),
                lambda: linear_adapted_backward(dy, x, w, a, index, saved), lambda: linear_adapted_backward(dy, x, w_t, a, index, saved[:, :, :16]),
                lambda: linear_adapted_backward(dy[:, :128], x, w_t, a, index, saved)):
        with pytest.raises(AssertionError):
            bad()
    odd = Adapters.from_weights(down[:, :, :120], up, scales)
    with pytest.raises(B.CascadeAttnError):
        linear_adapted(x[:, :120], w[:, :120], odd, index)
    odd = Adapters.from_weights(down, up[:, :200], scales)
    with pytest.raises(B.CascadeAttnError):                          # columns in whole steps of 128 for the way back
        linear_adapted_backward(dy[:, :200], x, w_t[:, :200], odd, index, saved)


def test_arguments_refused():
    """On the host, before anything is launched"""
    p = 4096
    good = dict(x=p, w=p, down=p, up=p, scales=p, index=p, low=p, y=p, m=600, n=136, k=256, adapters=3, rank=32, ldx=256, ldw=256, ldy=136, work=0, nbytes=0)
    for change, code in ((dict(m=-1), B.CA_EINVAL), (dict(adapters=0), B.CA_EINVAL), (dict(adapters=4097), B.CA_EUNSUPPORTED), (dict(rank=16), B.CA_EUNSUPPORTED),
                         (dict(rank=96), B.CA_EUNSUPPORTED), (dict(n=4), B.CA_EUNSUPPORTED), (dict(n=132), B.CA_EUNSUPPORTED), (dict(k=192), B.CA_EUNSUPPORTED),
                         (dict(n=2 ** 20 + 8, ldy=2 ** 20 + 8), B.CA_EUNSUPPORTED), (dict(m=2 ** 27 + 1), B.CA_EUNSUPPORTED), (dict(ldx=248), B.CA_EINVAL),
                         (dict(ldw=260), B.CA_EINVAL), (dict(ldx=2 ** 22), B.CA_EUNSUPPORTED), (dict(ldy=128), B.CA_EINVAL), (dict(ldy=140), B.CA_EINVAL),
                         (dict(scales=0), B.CA_EINVAL), (dict(index=0), B.CA_EINVAL), (dict(index=p + 2), B.CA_EINVAL), (dict(scales=p + 1), B.CA_EINVAL)) + tuple(
                             (dict([(name, at)]), B.CA_EINVAL) for name in ("x", "w", "down", "up", "low", "y") for at in (0, p + 8)):
        with pytest.raises(B.CascadeAttnError) as e:
            B.layer_linear_adapted_bf16(*{**good, **change}.values())
        assert e.value.code == code, change
    B.layer_linear_adapted_bf16(*{**good, "m": 0, "x": 0, "y": 0}.values())
    room = B.layer_linear_adapted_workspace(32, 64)
    assert room > 0 and B.layer_linear_adapted_workspace(513, 64) == 0 and B.layer_linear_adapted_workspace(5, 48) == 0
    for change in (dict(work=0, nbytes=room), dict(work=p + 8, nbytes=room), dict(work=p, nbytes=room - 1)):
        with pytest.raises(B.CascadeAttnError):
            B.layer_linear_adapted_bf16(*{**good, "m": 32, "rank": 64, **change}.values())
    assert B.layer_linear_adapted_backward_workspace(40, 136, 256, 3, 32) == 0 and B.layer_linear_adapted_backward_workspace(40, 256, 256, 3, 33) == 0
    assert B.layer_linear_adapted_backward_workspace(40, 256, 2 ** 20, 64, 32) == 0
    need = B.layer_linear_adapted_backward_workspace(40, 256, 384, 3, 32)
    assert need > 0
    back = dict(dy=p, x=p, w_t=p, down=p, up=p, scales=p, index=p, low=p, dx=p, d_down=p, d_up=p, m=40, n=256, k=384, adapters=3, rank=32, used=5, lddy=256, ldx=384,
                ldw=256, lddx=384, work=p, nbytes=need)
    for change in (dict(dx=0, d_down=0, d_up=0), dict(used=0), dict(used=33), dict(lddy=248), dict(ldx=380), dict(ldw=255), dict(lddx=376), dict(work=0),
                   dict(work=p + 4), dict(nbytes=need - 1), dict(dy=0), dict(x=0), dict(w_t=0), dict(down=0), dict(up=p + 8), dict(low=p + 8), dict(index=0),
                   dict(scales=0), dict(d_down=p + 1), dict(d_up=p + 1), dict(dx=p + 8)):
        with pytest.raises(B.CascadeAttnError) as e:
            B.layer_linear_adapted_backward_bf16(*{**back, **change}.values())
        assert e.value.code == B.CA_EINVAL, change
