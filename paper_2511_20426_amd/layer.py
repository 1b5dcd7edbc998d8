"""A whole layer of a video DiT around the cascaded attention, as a server runs it, and the training of its feed-forward half.

    y = x + W_out attention(rope(norm(q)), rope(norm(k)), v),  q | k | v = W_qkv x        z = y + W_down (act(W_gate y) * (W_up y))

The projections into and out of the attention and out of the feed-forward block are held and multiplied in 8 bits (linear_i8), gate and up
projection are one kernel in bf16 (gated_linear), queries and keys are normed per head on the way to their rotation, the keys on the way into
the shared pool.  Norms of the layer's input, modulation by the timestep and cross-attention are the caller's.  (Sizes are Wan's; its published
layers norm queries and keys over the whole width and have a plain gelu feed-forward half.)

Run as a program it times such a layer in the steady state of a cascade, or a training step of the feed-forward half:

    python -m paper_2511_20426_amd.layer                  # Wan-1.3B shape, five blocks in flight over six cached ones
    python -m paper_2511_20426_amd.layer --train          # gated projections and the one behind them, forward, backward, update
"""
from __future__ import annotations

import argparse
import json
from dataclasses import dataclass
from typing import Sequence

import torch

from . import binding as B
from .runner import CascadePool, QuantizedRows, gated_linear, gated_linear_backward, gated_linear_train, linear, linear_i8, quantize_rows


@dataclass
class CascadeLayer:
    """The weights of a layer: w_qkv [3 * width, width] with output rows ordered (q|k|v, head, dim), w_out [width, width], w_down [width, F] in 8
    bits, w_gate and w_up [F, width] in bf16, q_norm and k_norm [D]."""
    w_qkv: QuantizedRows
    w_out: QuantizedRows
    w_down: QuantizedRows
    w_gate: torch.Tensor
    w_up: torch.Tensor
    q_norm: torch.Tensor
    k_norm: torch.Tensor
    activation: str = "silu"
    eps: float = 1e-6

    @classmethod
    def from_weights(cls, w_qkv, w_out, w_gate, w_up, w_down, q_norm, k_norm, **more) -> "CascadeLayer":
        """From weights in bf16 or fp32: those that are held in 8 bits are brought to them, a scale for each output channel."""
        return cls(quantize_rows(w_qkv), quantize_rows(w_out), quantize_rows(w_down), w_gate, w_up, q_norm, k_norm, **more)

    def __call__(self, pool: CascadePool, x: torch.Tensor, inflight: Sequence[int], timesteps: Sequence[int], epoch: int = 0,
                 mode: int = B.CA_BIDIRECTIONAL) -> torch.Tensor:
        """One iteration for the blocks in flight (oldest first, consecutive in the video): x [C*L, width] -> [C*L, width]."""
        L, H, D = pool.block_tokens, pool.heads, pool.head_dim
        n = len(inflight) * L
        assert x.shape == (n, H * D) and all(b == inflight[0] + i for i, b in enumerate(inflight))
        qkv = linear_i8(x, self.w_qkv).view(n, 3, H, D)
        blocks = [qkv[i * L:(i + 1) * L] for i in range(len(inflight))]
        pool.append_batch(inflight, timesteps, epoch, [b[:, 1] for b in blocks], [b[:, 2] for b in blocks], k_weight=self.k_norm, eps=self.eps)
        q, _ = pool.qk_norm_rope(qkv[:, 0], None, self.q_norm, None, pool.frames_per_block * inflight[0], eps=self.eps)
        o = pool.forward(q, inflight, mode)
        x = x + linear_i8(o.view(n, H * D), self.w_out)
        h = gated_linear(x, self.w_gate, self.w_up, self.activation)
        return x + linear_i8(h, self.w_down)


def feed_forward_step(x, w_gate, w_up, w_down, target, activation: str = "silu", lr: float = 0.0):
    """One step of training the feed-forward half towards target [M, N] (mean squared error), all in bf16: (loss, gradients of w_gate, w_up,
    w_down and x); with lr the weights are updated in place.  (w_down, dy and h are transposed by torch's copies for the linear map, which multiplies
    rows by rows.)"""
    h, saved = gated_linear_train(x, w_gate, w_up, activation)
    y = linear(h, w_down)
    off = y.float() - target.float()
    dy = (off * (2.0 / off.numel())).to(torch.bfloat16)
    dh = linear(dy, w_down.t().contiguous())
    rows = -(-dy.shape[0] // 128) * 128                   # the linear map's k is whole steps of 128
    dyt, ht = (torch.zeros((t.shape[1], rows), dtype=t.dtype, device=t.device) for t in (dy, h))
    dyt[:, :dy.shape[0]], ht[:, :h.shape[0]] = dy.t(), h.t()
    dw_down = linear(dyt, ht)
    dx, dw_gate, dw_up = gated_linear_backward(dh, x, w_gate, w_up, saved, activation)
    if lr:
        for w, d in ((w_gate, dw_gate), (w_up, dw_up), (w_down, dw_down)):
            w.add_(d, alpha=-lr)
    return off.square().mean(), (dw_gate, dw_up, dw_down, dx)


def _timed(f, steps):
    for _ in range(3):
        f()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(steps):
        f()
    end.record()
    torch.cuda.synchronize()
    return start.elapsed_time(end) / steps


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--heads", type=int, default=12)
    p.add_argument("--grid", type=int, nargs=2, default=(30, 52), metavar=("H", "W"))
    p.add_argument("--inflight", type=int, default=5)
    p.add_argument("--cached", type=int, default=6)
    p.add_argument("--hidden", type=int, help="columns of the feed-forward block (8/3 of the width)")
    p.add_argument("--steps", type=int, default=10)
    p.add_argument("--train", action="store_true")
    a = p.parse_args()
    dev, width = "cuda:0", a.heads * 128
    hidden = a.hidden or -(-width * 8 // 3 // 128) * 128
    gen = torch.Generator(device=dev).manual_seed(0)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=gen, device=dev) * scale).to(torch.bfloat16)

    L = 3 * a.grid[0] * a.grid[1]
    w_gate, w_up, w_down = normal(hidden, width, scale=width ** -0.5), normal(hidden, width, scale=width ** -0.5), normal(width, hidden, scale=hidden ** -0.5)
    if a.train:
        x, target = normal(L, width), normal(L, width)
        losses = []
        ms = _timed(lambda: losses.append(feed_forward_step(x, w_gate, w_up, w_down, target, lr=64.0)[0]), a.steps)
        print(json.dumps({"metric": "feed_forward_training_step_ms", "value": ms, "rows": L, "width": width, "hidden": hidden,
                          "loss_first": losses[0].item(), "loss_last": losses[-1].item(), "data": "synthetic"}))
        return
    pool = CascadePool(heads=a.heads, head_dim=128, frames_per_block=3, grid_h=a.grid[0], grid_w=a.grid[1], rope_dims=(44, 42, 42), rope_theta=10000.0,
                       sink_blocks=0, window_blocks=a.cached, max_inflight=a.inflight, page_tokens=128, dtype="bf16", device=dev)
    layer = CascadeLayer.from_weights(normal(3 * width, width, scale=width ** -0.5), normal(width, width, scale=width ** -0.5), w_gate, w_up, w_down,
                                      normal(128), normal(128))
    for g in range(a.cached):
        pool.append(g, 0, 0, normal(L, a.heads, 128), normal(L, a.heads, 128))
        pool.ctx.kv_cache_promote(g)
    ids, x = list(range(a.cached, a.cached + a.inflight)), normal(a.inflight * L, width)
    ms = _timed(lambda: layer(pool, x, ids, [0] * a.inflight), a.steps)
    print(json.dumps({"metric": "layer_iteration_ms", "value": ms, "heads": a.heads, "width": width, "hidden": hidden, "tokens_per_block": L,
                      "inflight": a.inflight, "cached": a.cached, "data": "synthetic"}))


if __name__ == "__main__":
    main()
