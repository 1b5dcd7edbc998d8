"""The operators that a layer is adapted with, as they are used together: a modulated layer, an attention layer with adapters, the training of adapters
and the norm ahead of them by AdamW, of the feed-forward half by AdamW, and their commands."""
import json
import os
import shutil
import subprocess
import sys

import pytest
import torch

DEV = "cuda:0"


def _gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def _normal(gen, *shape, scale=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=gen, dtype=torch.float64) * scale).to(dtype).to(DEV)


def _pool(heads=2, grid=(4, 5), inflight=3):
    from paper_2511_20426_amd.runner import CascadePool
    return CascadePool(heads=heads, head_dim=128, frames_per_block=3, grid_h=grid[0], grid_w=grid[1], rope_dims=(44, 42, 42), rope_theta=10000.0,
                       sink_blocks=0, window_blocks=2, max_inflight=inflight, page_tokens=128, dtype="bf16")


@pytest.mark.gpu
def test_a_modulated_layer():
    """With weights of one and biases of zero it is the layer of the normed input; with gates of zero it leaves x as it is; each block goes by its own"""
    from paper_2511_20426_amd.layer import CascadeLayer
    from paper_2511_20426_amd.runner import layer_norm
    gen, width, hidden = _gen(0), 256, 384
    layer = CascadeLayer.from_weights(*(_normal(gen, *s, scale=s[1] ** -0.5) for s in ((3 * width, width), (width, width), (hidden, width), (hidden, width),
                                                                                         (width, hidden))), _normal(gen, 128), _normal(gen, 128))
    pools = [_pool() for _ in range(2)]
    L, ids = pools[0].block_tokens, [0, 1, 2]
    x = _normal(gen, 3 * L, width)
    mod = torch.zeros((3, 6, width), device=DEV)
    assert torch.equal(layer(pools[0], x, ids, [0] * 3, modulation=mod), x)
    mod[:, 0], mod[:, 2], mod[:, 3] = 1, 1, 1                        # the attention's half alone
    y = layer(pools[0], x, ids, [0] * 3, modulation=mod)
    normed = layer_norm(x, eps=1e-6)
    plain = CascadeLayer(layer.w_qkv, layer.w_out, layer.w_down, 0 * layer.w_gate, layer.w_up, layer.q_norm, layer.k_norm)        # no feed-forward part
    attended = plain(pools[1], normed, ids, [0] * 3).double() - normed.double()
    # both results are rounded to bf16 behind the same sum of a row and the same projection; attended is what is left of one of them
    assert ((y.double() - x.double() - attended).abs() <= 2.0 ** -8 * (y.double().abs() + 2 * (attended + normed.double()).abs() + attended.abs())).all()
    # another block's modulation changes nothing of the feed-forward half of the others: there tokens do not meet
    mod[:, 2] = 0
    mod[:, 5] = _normal(gen, 3, width, dtype=torch.float32)
    mod[:, 4] = _normal(gen, 3, width, dtype=torch.float32)
    one = layer(pools[0], x, ids, [0] * 3, modulation=mod)
    mod[1] = _normal(gen, 6, width, dtype=torch.float32)
    mod[1, 2] = 0
    two = layer(pools[0], x, ids, [0] * 3, modulation=mod)
    same = (one == two).view(3, L, width).flatten(1).all(1)
    assert same.tolist() == [True, False, True]


@pytest.mark.gpu
def test_an_attention_layer_with_adapters():
    """What the calls give one by one; rows without an adapter have the bits of the projection without them"""
    from paper_2511_20426_amd.runner import Adapters, attention_layer, linear, linear_adapted
    gen, H, D = _gen(1), 2, 128
    width, pools = H * D, [_pool(), _pool(), _pool()]
    L, ids = pools[0].block_tokens, [0, 1, 2]
    n = 3 * L
    x, w_qkv, w_out = _normal(gen, n, width), _normal(gen, 3 * width, width, scale=width ** -0.5), _normal(gen, width, width, scale=width ** -0.5)
    qkv = Adapters.from_weights(_normal(gen, 2, 8, width, scale=0.1), _normal(gen, 2, 3 * width, 8, scale=0.1), torch.tensor([1.0, 0.5], device=DEV))
    out = Adapters.from_weights(_normal(gen, 2, 8, width, scale=0.1), _normal(gen, 2, width, 8, scale=0.1))
    index = torch.tensor([0, 1, -1], dtype=torch.int32, device=DEV).repeat_interleave(L)
    y = attention_layer(pools[0], x, w_qkv, w_out, ids, [0] * 3, 0, 0, qkv_adapters=qkv, out_adapters=out, adapter_index=index)
    packed = linear_adapted(x, w_qkv, qkv, index)
    assert torch.equal(packed[2 * L:], linear(x[2 * L:], w_qkv)) and not torch.equal(packed[:L], linear(x[:L], w_qkv))
    parts = packed.view(n, 3, H, D)
    pools[1].append_batch(ids, [0] * 3, 0, [parts[i * L:(i + 1) * L, 1] for i in range(3)], [parts[i * L:(i + 1) * L, 2] for i in range(3)])
    o = pools[1].forward_rope(parts[:, 0], ids, 0)
    assert torch.equal(y, linear_adapted(o.view(n, width), w_out, out, index))
    none = torch.full_like(index, -1)
    assert torch.equal(attention_layer(pools[2], x, w_qkv, w_out, ids, [0] * 3, 0, 0, qkv_adapters=qkv, out_adapters=out, adapter_index=none),
                       attention_layer(pools[1], x, w_qkv, w_out, ids, [0] * 3, 0, 0))
    with pytest.raises(AssertionError):
        attention_layer(pools[2], x, w_qkv, w_out, ids, [0] * 3, 0, 0, publish_in_projection=True, qkv_adapters=qkv, adapter_index=index)


def _set(m, k, n, g, r, seed=2):
    gen = _gen(seed)
    x, w, target = _normal(gen, m, k), _normal(gen, n, k, scale=k ** -0.5), _normal(gen, m, n)
    down, up = _normal(gen, g, r, k, scale=k ** -0.5), _normal(gen, g, n, r, scale=0.3 * r ** -0.5)
    weight, bias = 1 + 0.1 * _normal(gen, k, dtype=torch.float32), 0.1 * _normal(gen, k, dtype=torch.float32)
    index = torch.randint(-1, g, (m,), generator=gen).to(torch.int32).to(DEV)
    return x, weight, bias, w, w.t().contiguous(), down, up, index, target


@pytest.mark.gpu
@pytest.mark.parametrize("m", [20, 333])
def test_a_step_of_training_adapters(m):
    """Loss and gradients of the whole against those of the formula in 64 bits, by their norms: on the way h, T, y, dy, dT and dh are rounded to bf16
    (2^-8 / sqrt(3) of a value in the mean at most), and each gradient once more: seven roundings, added as what is independent of one another."""
    from paper_2511_20426_amd.layer import adapter_step
    from paper_2511_20426_amd.optim import AdamW
    from paper_2511_20426_amd.runner import Adapters
    x, weight, bias, w, w_t, down, up, index, target = _set(m, 256, 384, 3, 32)
    adapters = Adapters.from_weights(down, up)
    masters = [down.float(), up.float(), weight, bias]
    optimizer = AdamW(masters, lr=1e-2, copies=(adapters.down, adapters.up, None, None))
    keep = [t.clone() for t in masters]
    args = [t.double().cpu().requires_grad_() for t in (down, up, weight, bias, x)]
    loss, grads = adapter_step(x, weight, bias, w, w_t, adapters, index, target, optimizer)
    d, u, wt, b, xd = args
    h = torch.nn.functional.layer_norm(xd, (256,), wt, b, 1e-6)
    y = h @ w.double().cpu().T
    for g in range(3):
        of = (index.cpu() == g).double()[:, None]
        y = y + of * ((h @ d[g].T) @ u[g].T)
    ref = ((y - target.double().cpu()) ** 2).mean()
    refs = torch.autograd.grad(ref, args)
    bound = (7 / 3) ** 0.5 * 2.0 ** -8
    assert abs(loss.item() - ref.item()) <= bound * ref.item()
    for got, want in zip(grads, refs):
        assert (got.double().cpu() - want).norm() <= bound * want.norm()
    # the step: by those gradients, into the masters and the adapters' own weights; a first step moves by lr g / (|g| + eps)
    for p, old, g in zip(masters, keep, grads):
        g = g.double()
        want = old.double() * (1 - 1e-4) - 1e-2 * g / (g.abs() + 1e-8)
        assert ((p.double() - want).abs() <= 2.0 ** -20 * (want.abs() + 1e-2)).all()
    assert torch.equal(adapters.down, masters[0].bfloat16()) and torch.equal(adapters.up, masters[1].bfloat16()) and optimizer.steps.tolist() == [1] * 4


@pytest.mark.gpu
def test_training_adapters_captured():
    """Forward, backward and step as one graph, replayed: the bits of as many eager steps"""
    from paper_2511_20426_amd.layer import adapter_step
    from paper_2511_20426_amd.optim import AdamW
    from paper_2511_20426_amd.runner import Adapters
    runs = []
    for _ in range(2):
        x, weight, bias, w, w_t, down, up, index, target = _set(150, 256, 384, 2, 32)
        adapters = Adapters.from_weights(down, up)
        masters = [down.float(), up.float(), weight, bias]
        optimizer = AdamW(masters, lr=1e-2, copies=(adapters.down, adapters.up, None, None))
        runs.append((masters, lambda s=(x, weight, bias, w, w_t, adapters, index, target, optimizer): adapter_step(*s)))
    (captured, one), (eager, other) = runs
    one()
    other()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for trip in range(4):
        graph.replay()
        other()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(captured, eager)), trip


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_of_the_feed_forward_half(bits):
    from paper_2511_20426_amd.layer import feed_forward_step
    from paper_2511_20426_amd.optim import AdamW
    gen, m, width, hidden = _gen(3), 130, 256, 384
    x, target = _normal(gen, m, width), _normal(gen, m, width)
    weights = [_normal(gen, *s, scale=s[1] ** -0.5) for s in ((hidden, width), (hidden, width), (width, hidden))]
    twins = [w.clone() for w in weights]
    optimizer = AdamW(weights, lr=1e-2, state_bits=bits)
    _, grads = feed_forward_step(x, *weights, target, optimizer=optimizer)
    _, same = feed_forward_step(x, *twins, target)
    again = AdamW(twins, lr=1e-2, state_bits=bits)
    again.step(same[:3])
    assert all(torch.equal(p, q) for p, q in zip(grads, same)) and all(torch.equal(p, q) for p, q in zip(weights, twins))


@pytest.mark.gpu
@pytest.mark.parametrize("args,metric", [(["--train", "--adamw", "8"], "feed_forward_training_step_ms"), (["--adapt", "--adapters", "3"], "adapter_training_step_ms")])
def test_commands(args, metric):
    r = subprocess.run([sys.executable, "-m", "paper_2511_20426_amd.layer", "--heads", "2", "--grid", "4", "5", "--steps", "2", *args], capture_output=True, text=True,
                       timeout=100)
    assert r.returncode == 0, r.stderr[-2000:]
    said = json.loads(r.stdout.strip().splitlines()[-1])
    assert said["metric"] == metric and said["value"] > 0 and said["loss_last"] == said["loss_last"]


def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc, exe = os.path.join(root, "paper_2511_20426_amd", "csrc"), str(tmp_path / "adapt_sanitize")
    subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
                    "-I", os.path.join(root, "include"), "-I", csrc, os.path.join(root, "tests", "adapt_sanitize_driver.cpp"),
                    os.path.join(csrc, "ca_adapt.cpp"), "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
                                                                                 UBSAN_OPTIONS="print_stacktrace=1"))
    assert r.returncode == 0 and "adapt sanitizer driver: ok" in r.stdout, r.stdout + r.stderr
