"""Torch plumbing around the C ABI: device memory for the pool and the current HIP stream.

No arithmetic of the method happens here; every tensor handed to the library is passed as a
raw device address.  Results carry no autograd history, whatever the arguments require: where there is a
backward pass (qk_norm_rope_backward, gated_linear_backward) the caller calls it.
"""
from __future__ import annotations

from typing import Sequence

import torch

from . import binding as B


# Small calls are bound by the host: a call whose arguments are all as they should be is taken by the extension (binding.calls), which
# checks them and calls the library.  What it does not take (it returns None then) goes on in Python, which raises or, for
# instance for integers of numpy, converts.  In the checks below a tensor's shape and strides are read once, as tuples, and no
# ctypes object is made for an address, for each look or object costs 0.1 us.
_BF16 = torch.bfloat16


def torch_dtype(dtype: str):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]


def _current_stream(device: torch.device) -> int:
    """Handle of the calling thread's current HIP stream on `device`.  (torch.cuda.current_stream builds a Stream
    object around it: 2.0 us of the 8.3 a small call takes, against 0.1.)"""
    index = device.index
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if index is None else index)


def _reachable(t: torch.Tensor, like: torch.Tensor) -> bool:
    """t's memory is there for a kernel that works on `like`: the same device's, or pinned host memory."""
    return t.device == like.device or t.is_pinned()


class CascadePool:
    """A ca_ctx over a pool tensor allocated with torch on the current device."""

    def __init__(self, *, heads, head_dim, frames_per_block, grid_h, grid_w, rope_dims, rope_theta,
                 sink_blocks, window_blocks, max_inflight, page_tokens, dtype, device="cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("CascadePool needs a GPU; use binding.Context(cfg) for metadata-only work")
        self.dtype = dtype
        self.device = torch.device(device)
        self.cfg = B.make_config(heads=heads, head_dim=head_dim, frames_per_block=frames_per_block,
                                 grid_h=grid_h, grid_w=grid_w, rope_dims=rope_dims, rope_theta=rope_theta,
                                 sink_blocks=sink_blocks, window_blocks=window_blocks,
                                 max_inflight=max_inflight, page_tokens=page_tokens, dtype=dtype)
        nbytes = B.pool_bytes(self.cfg)
        if nbytes == 0:
            raise ValueError("configuration rejected by ca_pool_bytes")
        self.pool = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.ctx = B.Context(self.cfg, self.pool.data_ptr(), nbytes)
        self.block_tokens = frames_per_block * grid_h * grid_w
        self.frames_per_block = frames_per_block
        self.heads, self.head_dim = heads, head_dim
        self._torch_dtype = torch_dtype(dtype)
        index = self.device.index
        self._shape = (heads, head_dim, self.block_tokens, int(dtype == "f32"), -1 if index is None else index)

    @classmethod
    def for_workload(cls, w, device="cuda:0"):
        return cls(heads=w.heads, head_dim=w.head_dim, frames_per_block=w.frames_per_block,
                   grid_h=w.grid_h, grid_w=w.grid_w, rope_dims=w.rope_dims, rope_theta=w.rope_theta,
                   sink_blocks=w.sink_blocks, window_blocks=max(w.window_blocks, w.n_cached - w.sink_blocks),
                   max_inflight=w.max_inflight, page_tokens=w.page_tokens, dtype=w.dtype, device=device)

    def _stream(self) -> int:
        return _current_stream(self.device)

    def _check(self, t: torch.Tensor) -> None:
        shape = t.shape
        assert t.is_cuda and t.dtype == self._torch_dtype and len(shape) == 3 and t.stride(2) == 1
        assert shape[1] == self.heads and shape[2] == self.head_dim

    def append(self, block_id: int, timestep: int, epoch: int, k: torch.Tensor, v: torch.Tensor) -> int:
        self._check(k); self._check(v)
        assert k.shape[0] == self.block_tokens and k.stride() == v.stride() and k.shape == v.shape
        return self.ctx.kv_cache_append(block_id, timestep, epoch, k.data_ptr(), v.data_ptr(),
                                        k.stride(0), k.stride(1), self._stream())

    def append_batch(self, block_ids: Sequence[int], timesteps: Sequence[int], epoch: int,
                     ks: Sequence[torch.Tensor], vs: Sequence[torch.Tensor], k_weight: torch.Tensor | None = None,
                     eps: float = 1e-6) -> list[int]:
        """All blocks of one cascade iteration in one launch; the tensors share their strides.  With k_weight [D] each head of K
        is normed (as qk_norm_rope does) ahead of its rotation."""
        h = self.ctx._h
        if h:
            r = (B.calls.append_batch(h.value, self._shape, block_ids, timesteps, epoch, ks, vs) if k_weight is None else
                 B.calls.append_batch_norm(h.value, self._shape, block_ids, timesteps, epoch, ks, vs, k_weight, eps))
            if r.__class__ is list:
                return r
            if r is not None:
                B._check(r, "kv_cache_append_batch" if k_weight is None else "kv_cache_append_batch_norm")
        stride = ks[0].stride()
        for k, v in zip(ks, vs):
            self._check(k); self._check(v)
            assert k.shape[0] == self.block_tokens and k.shape == v.shape
            assert k.stride() == stride and v.stride() == stride
        if k_weight is not None:
            self._check_weight(k_weight)
            return self.ctx.kv_cache_append_batch_norm(list(block_ids), list(timesteps), epoch, [k.data_ptr() for k in ks],
                                                       [v.data_ptr() for v in vs], stride[0], stride[1], k_weight.data_ptr(), eps,
                                                       self._stream())
        return self.ctx.kv_cache_append_batch(list(block_ids), list(timesteps), epoch,
                                              [k.data_ptr() for k in ks], [v.data_ptr() for v in vs],
                                              stride[0], stride[1], self._stream())

    def rope(self, x: torch.Tensor, first_frame: int, out: torch.Tensor | None = None) -> torch.Tensor:
        """Rotate x [n, H, D] (any token / head strides) into `out` (its own strides; default: a new
        contiguous tensor).  x is out is allowed."""
        h = self.ctx._h
        if h:
            r = B.calls.rope(h.value, self._shape, x, first_frame, out)
            if r.__class__ is int:
                B._check(r, "rope3d_apply_strided")
            if r is not None:
                return r
        self._check(x)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        self._check(y)
        assert y.shape == x.shape
        sx, sy = x.stride(), y.stride()
        self.ctx.rope3d_apply_strided(x.data_ptr(), sx[0], sx[1], y.data_ptr(), sy[0], sy[1], x.shape[0], first_frame,
                                      self._stream())
        return y

    def forward(self, q_rot: torch.Tensor, inflight: Sequence[int], mode: int,
                out: torch.Tensor | None = None, share: tuple[int, int] | None = None,
                static_scratch: bool = False) -> torch.Tensor:
        """Attention of the in-flight blocks' queries; with share = (first, count) only of blocks
        first .. first+count-1 of `inflight` (q_rot and the result then hold just those);
        static_scratch: through cascade_attn_forward_static (`out` must then be given: that call
        is for callers that do not allocate)."""
        h = self.ctx._h
        if h and not static_scratch:
            r = B.calls.forward(h.value, self._shape, q_rot, inflight, mode, out, share)
            if r.__class__ is int:
                B._check(r, "cascade_attn_forward" if share is None else "cascade_attn_forward_share")
            if r is not None:
                return r
        self._check(q_rot)
        n_q = len(inflight) if share is None else share[1]
        assert q_rot.is_contiguous() and q_rot.shape[0] == n_q * self.block_tokens
        o = torch.empty_like(q_rot) if out is None else out
        assert o.is_contiguous() and o.shape == q_rot.shape and o.dtype == q_rot.dtype and _reachable(o, q_rot)
        if static_scratch:
            assert share is None and out is not None
            self.ctx.cascade_attn_forward_static(q_rot.data_ptr(), list(inflight), mode, o.data_ptr(), self._stream())
        elif share is None:
            self.ctx.cascade_attn_forward(q_rot.data_ptr(), list(inflight), mode, o.data_ptr(), self._stream())
        else:
            self.ctx.cascade_attn_forward_share(q_rot.data_ptr(), list(inflight), share[0], share[1], mode,
                                                o.data_ptr(), self._stream())
        return o


def _forward_rope(self, q_raw: torch.Tensor, inflight: Sequence[int], mode: int,
                  out: torch.Tensor | None = None) -> torch.Tensor:
    """Attention on queries that are not rotated yet (cascade_attn_forward_rope): q_raw [C*L, H, D]
    with any token / head strides; the result is a contiguous tensor of that shape."""
    h = self.ctx._h
    if h:
        r = B.calls.forward_rope(h.value, self._shape, q_raw, inflight, mode, out)
        if r.__class__ is int:
            B._check(r, "cascade_attn_forward_rope")
        if r is not None:
            return r
    self._check(q_raw)
    assert q_raw.shape[0] == len(inflight) * self.block_tokens
    o = torch.empty(q_raw.shape, dtype=q_raw.dtype, device=q_raw.device) if out is None else out
    assert o.is_contiguous() and o.shape == q_raw.shape and o.dtype == q_raw.dtype and _reachable(o, q_raw)
    self.ctx.cascade_attn_forward_rope(q_raw.data_ptr(), q_raw.stride(0), q_raw.stride(1), list(inflight), mode,
                                       o.data_ptr(), self._stream())
    return o


CascadePool.forward_rope = _forward_rope


def _qkv_publish(self, x: torch.Tensor, w_qkv: torch.Tensor, block_ids: Sequence[int], timesteps: Sequence[int],
                 epoch: int, q_out: torch.Tensor | None = None) -> torch.Tensor:
    """QKV projection of the blocks in flight with their K/V published to the pool by the same
    launch (layer_qkv_publish); returns the packed, unrotated queries [C*L, H, D]."""
    h = self.ctx._h
    if h:
        r = B.calls.qkv_publish(h.value, self._shape, x, w_qkv, block_ids, timesteps, epoch, q_out)
        if r.__class__ is int:
            B._check(r, "layer_qkv_publish")
        if r is not None:
            return r
    n = len(block_ids) * self.block_tokens
    width = self.heads * self.head_dim
    assert x.is_cuda and x.dtype == torch.bfloat16 and x.dim() == 2 and x.shape[0] == n and x.stride(1) == 1
    assert w_qkv.shape == (3 * width, x.shape[1]) and w_qkv.stride(1) == 1 and w_qkv.dtype == torch.bfloat16 and _reachable(w_qkv, x)
    q = torch.empty((n, self.heads, self.head_dim), dtype=torch.bfloat16, device=x.device) if q_out is None else q_out
    assert q.is_contiguous() and q.shape == (n, self.heads, self.head_dim) and q.dtype == torch.bfloat16 and _reachable(q, x)
    self.ctx.layer_qkv_publish(list(block_ids), list(timesteps), epoch, x.data_ptr(), x.stride(0), w_qkv.data_ptr(),
                               w_qkv.stride(0), x.shape[1], q.data_ptr(), self._stream())
    return q


CascadePool.qkv_publish = _qkv_publish


def _check_weight(self, w: torch.Tensor) -> None:
    assert w.is_cuda and w.dtype == self._torch_dtype and w.shape == (self.head_dim,) and (self.head_dim == 1 or w.stride(0) == 1)


def _view(self, t: torch.Tensor, n: int):
    """(address, token stride, head stride) of a [n, H, D] tensor; of a single token or head the stride is free."""
    self._check(t)
    assert t.shape[0] == n
    s = t.stride()
    return (t.data_ptr(), s[0] if n > 1 else self.heads * self.head_dim, s[1] if self.heads > 1 else self.head_dim)


def _qk_norm_rope(self, q: torch.Tensor | None, k: torch.Tensor | None, q_weight: torch.Tensor | None, k_weight: torch.Tensor | None,
                  first_frame: int, eps: float = 1e-6, q_out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """Each head of q and k (either may be None) normed, y = weight * x / sqrt(mean(x^2) + eps), and rotated by its token's
    position, in one launch: [n, H, D] with any token / head strides, consecutive tokens from latent frame `first_frame` on; weights
    [D].  Returns (q', k'), in q_out / k_out (their own strides) or new contiguous tensors; an output may be its input."""
    h = self.ctx._h
    if h:
        r = B.calls.norm_rope(h.value, self._shape, q, k, q_weight, k_weight, first_frame, eps, q_out, k_out)
        if r.__class__ is int:
            B._check(r, "layer_qk_norm_rope")
        if r is not None:
            return r
    given, outs, views = [], [], []
    n = (k if q is None else q).shape[0]
    for x, w, out in ((q, q_weight, q_out), (k, k_weight, k_out)):
        if x is None:
            assert w is None and out is None
            views += [None, None]
            given.append(0)
            outs.append(None)
            continue
        self._check_weight(w)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device) if out is None else out
        views += [self._view(x, n), self._view(y, n)]
        given.append(w.data_ptr())
        outs.append(y)
    self.ctx.layer_qk_norm_rope(views[0], views[2], given[0], given[1], eps, views[1], views[3], n, first_frame, self._stream())
    return outs[0], outs[1]


def _qk_norm_rope_backward(self, dq_out: torch.Tensor | None, dk_out: torch.Tensor | None, q: torch.Tensor | None,
                           k: torch.Tensor | None, q_weight: torch.Tensor | None, k_weight: torch.Tensor | None, first_frame: int,
                           eps: float = 1e-6, dq: torch.Tensor | None = None, dk: torch.Tensor | None = None):
    """Gradients of qk_norm_rope: from those of its outputs (dq_out, dk_out) and its inputs to (dq, dk, dq_weight, dk_weight), the
    weights' in fp32.  What belongs to a q or k of None is None.  dq may be dq_out, dk dk_out."""
    h = self.ctx._h
    if h:
        r = B.calls.norm_rope_backward(h.value, self._shape, dq_out, dk_out, q, k, q_weight, k_weight, first_frame, eps, dq, dk)
        if r.__class__ is int:
            B._check(r, "layer_qk_norm_rope_backward")
        if r is not None:
            return r
    n = (k if q is None else q).shape[0]
    views, weights, grads, dws = [], [], [], []
    for x, w, dz, dx in ((q, q_weight, dq_out, dq), (k, k_weight, dk_out, dk)):
        if x is None:
            assert w is None and dz is None and dx is None
            views.append((None, None, None))
            weights.append(0)
            grads.append(None)
            dws.append(None)
            continue
        self._check_weight(w)
        g = torch.empty(x.shape, dtype=x.dtype, device=x.device) if dx is None else dx
        views.append((self._view(dz, n), self._view(x, n), self._view(g, n)))
        weights.append(w.data_ptr())
        grads.append(g)
        dws.append(torch.empty(self.head_dim, dtype=torch.float32, device=x.device))
    nbytes = self.ctx.layer_qk_norm_rope_workspace()
    work = torch.empty(nbytes, dtype=torch.uint8, device=(k if q is None else q).device)
    (dzq, xq, gq), (dzk, xk, gk) = views
    self.ctx.layer_qk_norm_rope_backward(dzq, dzk, xq, xk, weights[0], weights[1], eps, gq, gk, *(0 if d is None else d.data_ptr() for d in dws),
                                         n, first_frame, work.data_ptr(), nbytes, self._stream())
    return grads[0], grads[1], dws[0], dws[1]


CascadePool._check_weight = _check_weight
CascadePool._view = _view
CascadePool.qk_norm_rope = _qk_norm_rope
CascadePool.qk_norm_rope_backward = _qk_norm_rope_backward


def linear(x: torch.Tensor, w: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """y = x @ w.T through layer_linear_bf16: x [M, K], w [N, K], y [M, N], bf16, rows may be
    strided (last dimension contiguous)."""
    r = B.calls.linear(x, w, out)
    if r.__class__ is int:
        B._check(r, "layer_linear_bf16")
    if r is not None:
        return r
    assert x.is_cuda and w.is_cuda and x.dtype == _BF16 and w.dtype == _BF16
    xs, ws, sx, sw = x.shape, w.shape, x.stride(), w.stride()
    assert len(xs) == 2 and len(ws) == 2 and xs[1] == ws[1] and sx[1] == 1 and sw[1] == 1
    shape, device = (xs[0], ws[0]), x.device
    y = torch.empty(shape, dtype=_BF16, device=device) if out is None else out
    sy = y.stride()
    assert y.shape == shape and sy[1] == 1 and y.dtype == _BF16 and _reachable(y, x)
    B.layer_linear_bf16(x.data_ptr(), w.data_ptr(), y.data_ptr(), xs[0], ws[0], xs[1], sx[0], sw[0], sy[0],
                        _current_stream(device))
    return y


def _matrix(t: torch.Tensor, like: torch.Tensor, dtype, rows: int, cols: int) -> int:
    """The row stride of a [rows, cols] matrix with unit stride along its rows; that of a single row is free."""
    shape, s = t.shape, t.stride()
    assert t.dtype == dtype and len(shape) == 2 and shape[0] == rows and shape[1] == cols and (s[1] == 1 or cols == 1) and _reachable(t, like)
    return s[0] if rows > 1 else -(-cols // 16) * 16


class QuantizedRows:
    """Rows in 8 bits with a scale each (layer_quantize_rows_i8): codes [rows, k filled up with zeros to a multiple of 256] and
    scales [rows]; what they stand for is codes[:, :k] * scales[:, None]."""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, k: int):
        assert codes.dtype == torch.int8 and codes.dim() == 2 and codes.stride(1) == 1 and codes.shape[1] == -(-k // 256) * 256
        assert scales.dtype == torch.float32 and scales.shape == (codes.shape[0],) and scales.is_contiguous() and scales.device == codes.device
        self.codes, self.scales, self.k = codes, scales, k

    @property
    def shape(self):
        return (self.codes.shape[0], self.k)

    @classmethod
    def from_codes(cls, codes: torch.Tensor, scales: torch.Tensor) -> "QuantizedRows":
        """From codes [rows, k] and scales [rows] made elsewhere (a checkpoint's)."""
        rows, k = codes.shape
        if k % 256 == 0 and codes.dtype == torch.int8 and codes.stride(1) == 1 and codes.stride(0) % 16 == 0 and codes.data_ptr() % 16 == 0:
            whole = codes                          # as they are
        else:
            whole = torch.zeros((rows, -(-k // 256) * 256), dtype=torch.int8, device=codes.device)
            whole[:, :k] = codes
        return cls(whole, scales.to(torch.float32).contiguous(), k)


def quantize_rows(x: torch.Tensor) -> QuantizedRows:
    """x [rows, k], bf16 or fp32, in 8 bits: a scale of largest magnitude / 127 for each row, codes rounded half to even."""
    assert x.is_cuda and x.dim() == 2 and x.dtype in (torch.bfloat16, torch.float32)
    rows, k = x.shape
    ldx = _matrix(x, x, x.dtype, rows, k)
    codes = torch.empty((rows, -(-k // 256) * 256), dtype=torch.int8, device=x.device)
    scales = torch.empty(rows, dtype=torch.float32, device=x.device)
    B.layer_quantize_rows_i8(x.data_ptr(), B.CA_BF16 if x.dtype == _BF16 else B.CA_F32, codes.data_ptr(), scales.data_ptr(), rows, k, ldx,
                             codes.shape[1], _current_stream(x.device))
    return QuantizedRows(codes, scales, k)


def linear_i8(x: torch.Tensor | QuantizedRows, w: QuantizedRows, out: torch.Tensor | None = None) -> torch.Tensor:
    """y = x @ w.T in 8-bit integers with a scale for each row of x (token) and of w (output channel), y [M, N] in bf16; x [M, K] in bf16
    or fp32 is brought to 8 bits on the way."""
    r = B.calls.linear_i8(x, w.codes, w.scales, w.k, out)
    if r.__class__ is int:
        B._check(r, "layer_linear_i8_values")
    if r is not None:
        return r
    n, k, device = w.shape[0], w.k, w.codes.device
    assert w.codes.is_cuda
    m = x.shape[0]
    y = torch.empty((m, n), dtype=_BF16, device=device) if out is None else out
    ldw, ldy = w.codes.shape[1] if n <= 1 else w.codes.stride(0), _matrix(y, w.codes, _BF16, m, n)
    if isinstance(x, QuantizedRows):
        assert x.k == k and x.codes.device == device
        B.layer_linear_i8(x.codes.data_ptr(), x.scales.data_ptr(), w.codes.data_ptr(), w.scales.data_ptr(), y.data_ptr(), m, n, k,
                          x.codes.shape[1] if m <= 1 else x.codes.stride(0), ldw, ldy, _current_stream(device))
        return y
    assert x.is_cuda and x.device == device and x.dtype in (_BF16, torch.float32)
    ldx = _matrix(x, w.codes, x.dtype, m, k)
    nbytes = B.layer_linear_i8_workspace(m, k)
    work = torch.empty(nbytes, dtype=torch.uint8, device=device)
    B.layer_linear_i8_values(x.data_ptr(), B.CA_BF16 if x.dtype == _BF16 else B.CA_F32, w.codes.data_ptr(), w.scales.data_ptr(), y.data_ptr(), m, n,
                             k, ldx, ldw, ldy, work.data_ptr(), nbytes, _current_stream(device))
    return y


_ACTIVATIONS = {"silu": B.CA_SILU, "gelu": B.CA_GELU}


def _gated(x, w_gate, w_up, activation, out, saved):
    assert x.is_cuda and w_gate.is_cuda and w_up.is_cuda
    (m, k), f, device = x.shape, w_gate.shape[0], x.device
    ldx, ldg, ldu = _matrix(x, x, _BF16, m, k), _matrix(w_gate, x, _BF16, f, k), _matrix(w_up, x, _BF16, f, k)
    h = torch.empty((m, f), dtype=_BF16, device=device) if out is None else out
    B.layer_gated_bf16(x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), h.data_ptr(), 0 if saved is None else saved.data_ptr(),
                       _ACTIVATIONS[activation], m, f, k, ldx, ldg, ldu, _matrix(h, x, _BF16, m, f), _current_stream(device))
    return h


def gated_linear(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, activation: str = "silu",
                 out: torch.Tensor | None = None) -> torch.Tensor:
    """h = act(x @ w_gate.T) * (x @ w_up.T), the first half of a gated feed-forward block, in one kernel: x [M, K], w_gate and w_up
    [F, K], h [M, F], bf16, rows may be strided (last dimension contiguous); activation "silu" or "gelu" (its tanh form)."""
    r = B.calls.gated(x, w_gate, w_up, _ACTIVATIONS[activation], out, False)
    if r.__class__ is int:
        B._check(r, "layer_gated_bf16")
    return _gated(x, w_gate, w_up, activation, out, None) if r is None else r


def gated_linear_train(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, activation: str = "silu",
                       out: torch.Tensor | None = None):
    """gated_linear for training: (h, saved), saved being the two projections in fp32 as gated_linear_backward takes them (in an
    order of the library's own)."""
    r = B.calls.gated(x, w_gate, w_up, _ACTIVATIONS[activation], out, True)
    if r.__class__ is int:
        B._check(r, "layer_gated_bf16")
    if r is not None:
        return r
    saved = torch.empty(B.layer_gated_saved_bytes(x.shape[0], w_gate.shape[0]) // 4, dtype=torch.float32, device=x.device)
    return _gated(x, w_gate, w_up, activation, out, saved), saved


def gated_linear_backward(dh: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, saved: torch.Tensor,
                          activation: str = "silu"):
    """(dx, dw_gate, dw_up) from the gradient dh [M, F] of gated_linear_train's h, its inputs and what it saved."""
    r = B.calls.gated_backward(x, w_gate, w_up, dh, saved, _ACTIVATIONS[activation])
    if r.__class__ is int:
        B._check(r, "layer_gated_backward_bf16")
    if r is not None:
        return r
    assert x.is_cuda and w_gate.is_cuda and w_up.is_cuda
    (m, k), f, device = x.shape, w_gate.shape[0], x.device
    ldx, ldg, ldu = _matrix(x, x, _BF16, m, k), _matrix(w_gate, x, _BF16, f, k), _matrix(w_up, x, _BF16, f, k)
    lddh = _matrix(dh, x, _BF16, m, f)
    assert saved.dtype == torch.float32 and saved.numel() * 4 == B.layer_gated_saved_bytes(m, f) and saved.is_contiguous() and _reachable(saved, x)
    dx, dw = torch.empty((m, k), dtype=_BF16, device=device), torch.empty((2, f, k), dtype=_BF16, device=device)
    nbytes = B.layer_gated_backward_workspace(m, f, k)
    work = torch.empty(nbytes, dtype=torch.uint8, device=device)
    B.layer_gated_backward_bf16(dh.data_ptr(), x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), saved.data_ptr(),
                                _ACTIVATIONS[activation], dx.data_ptr(), dw[0].data_ptr(), dw[1].data_ptr(), m, f, k, lddh, ldx, ldg, ldu,
                                k, k, work.data_ptr(), nbytes, _current_stream(device))
    return dx, dw[0], dw[1]


def attention_layer(pool: CascadePool, x: torch.Tensor, w_qkv: torch.Tensor, w_out: torch.Tensor,
                    inflight: Sequence[int], timesteps: Sequence[int], epoch: int, mode: int,
                    rotate_q_in_kernel: bool = True, publish_in_projection: bool = False) -> torch.Tensor:
    """One self-attention layer around the shared pool, for the blocks in flight (oldest first,
    consecutive in the video): QKV projection, K/V of every block published to the cache, Q
    rotated, cascaded attention, output projection.  x [C*L, width], w_qkv [3*width, width] with
    output rows ordered (q|k|v, head, dim), w_out [width, width]; width = heads * head_dim.
    Library calls only; the q/k/v handed on are strided views of the projection's output.  The
    queries go to the attention kernel as they are (it rotates them while loading), or, with
    rotate_q_in_kernel=False, through rope3d_apply into a contiguous tensor first.  With
    publish_in_projection the first two steps are one launch (layer_qkv_publish): K/V go from the
    projection's epilogue straight into pool pages; three launches per layer in all."""
    L, H, D = pool.block_tokens, pool.heads, pool.head_dim
    n = len(inflight) * L
    assert x.shape == (n, H * D) and w_qkv.shape == (3 * H * D, H * D) and w_out.shape == (H * D, H * D)
    if publish_in_projection:
        q = pool.qkv_publish(x, w_qkv, inflight, timesteps, epoch)
        o = pool.forward_rope(q, inflight, mode)
        return linear(o.view(n, H * D), w_out)
    qkv = linear(x, w_qkv).view(n, 3, H, D)
    blocks = [qkv[i * L:(i + 1) * L] for i in range(len(inflight))]
    pool.append_batch(inflight, timesteps, epoch, [b[:, 1] for b in blocks], [b[:, 2] for b in blocks])
    if rotate_q_in_kernel:
        o = pool.forward_rope(qkv[:, 0], inflight, mode)
    else:
        q_rot = pool.rope(qkv[:, 0], pool.frames_per_block * inflight[0])     # strided view -> contiguous
        o = pool.forward(q_rot, inflight, mode)
    return linear(o.view(n, H * D), w_out)
