"""Python binding of include/heinsen_attention.h: the recurrence with a matrix state (attention with a decay for each
head), its one-token step, and the norms around a block built on it.

    S_t = exp(log_a_t) S_{t-1} + k_t v_t^T,   o_t = scale * S_t^T q_t

As in ``heinsen_scan`` every step of the computation runs in the library's CUDA kernels; PyTorch provides device memory,
streams and the autograd graph.  There is no CPU fallback.  ``decay_attention``, ``block_norms`` and ``gated_norm`` are
differentiable in every tensor argument (once: their gradients are not differentiable again).
"""
from __future__ import annotations

import ctypes

import torch

from .heinsen_scan import HeinsenScanError, _check, _dtype_code, _on_device, _ptr, _stream_ptr, lib as _scan_lib  # noqa: F401

EXPORTS = [
    "heinsen_attention_forward", "heinsen_attention_backward", "heinsen_attention_workspace_bytes",
    "heinsen_attention_step", "heinsen_block_norms_forward", "heinsen_block_norms_backward",
    "heinsen_block_norms_workspace_bytes", "heinsen_gated_norm_forward", "heinsen_gated_norm_backward",
    "heinsen_gated_norm_workspace_bytes",
]


class _Tensor(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class _Problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("tokens", ctypes.c_int64), ("heads", ctypes.c_int32), ("q_heads", ctypes.c_int32),
                ("k_heads", ctypes.c_int32), ("v_heads", ctypes.c_int32), ("k_dim", ctypes.c_int32), ("v_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int), ("scale", ctypes.c_float), ("q", _Tensor), ("k", _Tensor), ("v", _Tensor),
                ("log_a", _Tensor), ("state0", ctypes.c_void_p), ("lengths", ctypes.c_void_p)]


class _Norms(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("gate_rows", ctypes.c_int64), ("dim", ctypes.c_int32), ("dtype", ctypes.c_int),
                ("weight_dtype", ctypes.c_int), ("scale", ctypes.c_float), ("eps", ctypes.c_float), ("x", ctypes.c_void_p),
                ("branch", ctypes.c_void_p), ("gate", ctypes.c_void_p), ("pre_weight", ctypes.c_void_p),
                ("post_weight", ctypes.c_void_p)]


_lib = None


def lib() -> ctypes.CDLL:
    """The shared library, with the functions of heinsen_attention.h bound.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = _scan_lib()
        vp, sz, ci, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64
        pr, te, no = ctypes.POINTER(_Problem), ctypes.POINTER(_Tensor), ctypes.POINTER(_Norms)
        for name, args, res in (
                ("heinsen_attention_forward", [pr, te, vp, vp, sz, vp], ci),
                ("heinsen_attention_backward", [pr, te, vp, vp, vp, vp, vp, vp, vp, sz, vp], ci),
                ("heinsen_attention_workspace_bytes", [pr, ci], sz),
                ("heinsen_attention_step", [pr, te, vp, i64, vp, vp], ci),
                ("heinsen_block_norms_forward", [no, vp, vp, vp], ci),
                ("heinsen_block_norms_backward", [no, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp], ci),
                ("heinsen_block_norms_workspace_bytes", [no], sz),
                ("heinsen_gated_norm_forward", [no, vp, vp], ci),
                ("heinsen_gated_norm_backward", [no, vp, vp, vp, vp, vp, sz, vp], ci),
                ("heinsen_gated_norm_workspace_bytes", [no], sz)):
            getattr(L, name).argtypes, getattr(L, name).restype = args, res
        _lib = L
    return _lib


def _cuda(name: str, device=None, **tensors):
    for n, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError(f"{n} must be a CUDA tensor (there is no CPU path)")
        if device is not None and t.device != device:
            raise ValueError(f"{name}: {n} is on {t.device}, not on {device}")


def _space(nbytes: int, device) -> torch.Tensor:
    if nbytes == 0:
        raise ValueError("the library does not accept these sizes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _tensor(t: torch.Tensor, name: str) -> _Tensor:
    """[batch, tokens, heads, dim] of any strides, the last dimension contiguous."""
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return _Tensor(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def _state_ok(t, shape, name):
    if t is None:
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dtype != torch.float32:
        raise TypeError(f"{name} must be float32")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _problem(q, k, v, log_a, state0, scale, lengths) -> _Problem:
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v are [batch, tokens, heads, dim]")
    b, t, hq, kd = q.shape
    hk, hv, vd = k.shape[2], v.shape[2], v.shape[3]
    if k.shape[:2] != (b, t) or v.shape[:2] != (b, t) or k.shape[3] != kd:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k, v must share one dtype")
    if log_a.dtype != torch.float32:
        raise TypeError("log_a must be float32")
    if log_a.dim() == 1:
        h, la = log_a.shape[0], _Tensor(log_a.data_ptr(), 0, 0, log_a.stride(0))
    elif log_a.dim() == 3 and log_a.shape[:2] == (b, t):
        h, la = log_a.shape[2], _Tensor(log_a.data_ptr(), *log_a.stride())
    else:
        raise ValueError(f"log_a: expected shape [heads] or {(b, t, 'heads')}, got {tuple(log_a.shape)}")
    if any(n < 1 or h % n for n in (hq, hk, hv)):
        raise ValueError(f"the {h} heads of log_a must be a multiple of the heads of q ({hq}), k ({hk}) and v ({hv})")
    _state_ok(state0, (b, h, kd, vd), "state0")
    if lengths is not None and (lengths.dtype != torch.int32 or tuple(lengths.shape) != (b,) or not lengths.is_contiguous()):
        raise ValueError("lengths must be a contiguous int32 tensor [batch]")
    _cuda("decay_attention", q.device, q=q, k=k, v=v, log_a=log_a, state0=state0, lengths=lengths)
    return _Problem(b, t, h, hq, hk, hv, kd, vd, _dtype_code(q), scale, _tensor(q, "q"), _tensor(k, "k"), _tensor(v, "v"), la,
                    state0.data_ptr() if state0 is not None else None, lengths.data_ptr() if lengths is not None else None)


def _attention_forward(p: _Problem, q: torch.Tensor):
    dev = q.device
    o = torch.empty((p.batch, p.tokens, p.heads, p.v_dim), dtype=q.dtype, device=dev)
    state = torch.empty((p.batch, p.heads, p.k_dim, p.v_dim), dtype=torch.float32, device=dev)
    ws = _space(int(lib().heinsen_attention_workspace_bytes(p, 0)), dev)
    with _on_device(dev):
        _check(lib().heinsen_attention_forward(p, _tensor(o, "o"), _ptr(state), _ptr(ws), ws.numel(), _stream_ptr(dev)))
    return o, state


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_a, state0, scale, lengths):
        p = _problem(q, k, v, log_a, state0, scale, lengths)
        o, state = _attention_forward(p, q)
        ctx.save_for_backward(q, k, v, log_a, state0, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, state

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_o, d_state):
        q, k, v, log_a, state0, lengths = ctx.saved_tensors
        p = _problem(q, k, v, log_a, state0, ctx.scale, lengths)
        dev = q.device
        if d_o is None:
            d_o = torch.zeros((p.batch, p.tokens, p.heads, p.v_dim), dtype=q.dtype, device=dev)
        if d_o.shape[-1] > 1 and d_o.stride(-1) != 1:
            d_o = d_o.contiguous()
        if d_state is not None:
            d_state = d_state.contiguous()
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
        dla = torch.empty(log_a.shape, dtype=torch.float32, device=dev) if ctx.needs_input_grad[3] else None
        if dla is not None and log_a.dim() == 3 and log_a.stride(0) == 0 and log_a.stride(1) == 0 and p.tokens * p.batch:
            log_a = log_a.contiguous()  # an expanded [heads]: its gradient is still asked for every token
            p.log_a = _tensor(log_a, "log_a")
        ds0 = torch.empty(state0.shape, dtype=torch.float32, device=dev) if ctx.needs_input_grad[4] else None
        ws = _space(int(lib().heinsen_attention_workspace_bytes(p, 1)), dev)
        with _on_device(dev):
            _check(lib().heinsen_attention_backward(p, _tensor(d_o, "d_o"), _ptr(d_state), _ptr(dq), _ptr(dk), _ptr(dv),
                                                    _ptr(dla), _ptr(ds0), _ptr(ws), ws.numel(), _stream_ptr(dev)))
        return dq, dk, dv, dla, ds0, None, None


def decay_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor,
                    state0: torch.Tensor | None = None, *, scale: float | None = None,
                    lengths: torch.Tensor | None = None):
    """Attention with a decay for each head over whole sequences; returns (o, state).  Asynchronous, differentiable.

    q [B, T, Hq, K], k [B, T, Hk, K], v [B, T, Hv, V]: float32 or bfloat16, last dimension contiguous, any other strides;
    log_a: float32 [B, T, H], or [H] for fixed decays, H a multiple of Hq, Hk and Hv (head h reads head h * Hq // H of q);
    state0 [B, H, K, V] float32 continues earlier tokens; lengths [B] int32 ends row b after lengths[b] tokens.
    scale defaults to K ** -0.5.  o [B, T, H, V] has q's dtype, state [B, H, K, V] is float32 (what the next call or
    ``decay_attention_step`` takes).  log_a = -inf forgets the state at that token: packed sequences start so.
    """
    scale = float(q.shape[-1] ** -0.5 if scale is None else scale)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, v, log_a, state0)):
        return _DecayAttention.apply(q, k, v, log_a, state0, scale, lengths)
    return _attention_forward(_problem(q, k, v, log_a, state0, scale, lengths), q)


def decay_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor, state: torch.Tensor, *,
                         scale: float | None = None, slots: torch.Tensor | None = None,
                         out: torch.Tensor | None = None) -> torch.Tensor:
    """One token for each sequence: updates ``state`` in place and returns o [B, H, V].  Asynchronous, not differentiable.

    q [B, Hq, K], k [B, Hk, K], v [B, Hv, V]; log_a float32 [B, H] or [H]; state float32 [N, H, K, V], of which sequence b
    uses row slots[b] (int32; negative or >= N: no state, o is zero), or row b.  No two sequences may share a row.
    """
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k, v are [batch, heads, dim]")
    b, kd = q.shape[0], q.shape[2]
    la = log_a if log_a.dim() == 1 else log_a.unsqueeze(1)
    p = _problem(q.unsqueeze(1), k.unsqueeze(1), v.unsqueeze(1), la, None, float(kd ** -0.5 if scale is None else scale), None)
    _state_ok(state, (state.shape[0], p.heads, kd, p.v_dim), "state")
    if slots is None:
        if state.shape[0] < b:
            raise ValueError(f"state has {state.shape[0]} rows for {b} sequences")
    elif slots.dtype != torch.int32 or tuple(slots.shape) != (b,) or not slots.is_contiguous():
        raise ValueError("slots must be a contiguous int32 tensor [batch]")
    if out is None:
        out = torch.empty((b, p.heads, p.v_dim), dtype=q.dtype, device=q.device)
    elif tuple(out.shape) != (b, p.heads, p.v_dim) or out.dtype != q.dtype:
        raise ValueError("out must be [batch, heads, v_dim] of q's dtype")
    _cuda("decay_attention_step", q.device, state=state, slots=slots, out=out)
    with _on_device(q.device):
        _check(lib().heinsen_attention_step(p, _tensor(out.unsqueeze(1), "out"), _ptr(state), state.shape[0], _ptr(slots),
                                            _stream_ptr(q.device)))
    return out


# ------------------------------------------------------------------------------------------------------------- norms

def _norms_problem(name, x, weight, eps, scale=1.0, branch=None, gate=None, post=None) -> _Norms:
    dim = x.shape[-1]
    rows, gate_rows = x.numel() // dim if dim else 0, 1
    _dtype_code(x)
    for n, t in (("branch", branch),):
        if t is not None and (t.shape != x.shape or t.dtype != x.dtype):
            raise ValueError(f"{name}: {n} must have the shape and dtype of x")
    if gate is not None:
        if gate.dtype != x.dtype:
            raise TypeError(f"{name}: gate must have the dtype of x")
        if gate.shape != x.shape:
            # a gate for each sequence: [.., 1, dim] beside [.., tokens, dim]
            if branch is None or x.dim() < 2 or gate.shape != (*x.shape[:-2], 1, dim):
                raise ValueError(f"{name}: gate has shape {tuple(gate.shape)} beside {tuple(x.shape)}")
            gate_rows = x.shape[-2]
    for n, t in (("weight", weight), ("post_weight", post)):
        if t is not None and tuple(t.shape) != (dim,):
            raise ValueError(f"{name}: {n} must be [{dim}]")
        if t is not None and t.dtype != torch.float32 and t.dtype != x.dtype:
            raise TypeError(f"{name}: {n} must be float32 or of x's dtype")
    if post is not None and post.dtype != weight.dtype:
        raise TypeError(f"{name}: both weights must share one dtype")
    for n, t in (("x", x), ("branch", branch), ("gate", gate), ("weight", weight), ("post_weight", post)):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name}: {n} must be contiguous")
    _cuda(name, x.device, x=x, branch=branch, gate=gate, weight=weight, post_weight=post)
    ptr = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    return _Norms(rows, max(1, gate_rows), dim, _dtype_code(x), _dtype_code(weight), scale, eps, ptr(x), ptr(branch), ptr(gate),
                  ptr(weight), ptr(post))


def _block_norms_forward(p: _Norms, x):
    r, y = torch.empty_like(x), torch.empty_like(x)
    with _on_device(x.device):
        _check(lib().heinsen_block_norms_forward(p, _ptr(r), _ptr(y), _stream_ptr(x.device)))
    return r, y


class _BlockNorms(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, branch, pre, post, gate, scale, eps):
        p = _norms_problem("block_norms", x, pre, eps, scale, branch, gate, post)
        ctx.save_for_backward(x, branch, pre, post, gate)
        ctx.numbers = (eps, scale)
        ctx.set_materialize_grads(False)
        return _block_norms_forward(p, x)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_r, d_y):
        x, branch, pre, post, gate = ctx.saved_tensors
        eps, scale = ctx.numbers
        p = _norms_problem("block_norms", x, pre, eps, scale, branch, gate, post)
        d_y = torch.zeros_like(x) if d_y is None else d_y.contiguous()
        d_r = None if d_r is None else d_r.contiguous()
        new = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
        dx, dh, dpre, dpost, dgate = new(x), new(branch), new(pre), new(post), new(gate)
        ws = _space(int(lib().heinsen_block_norms_workspace_bytes(p)), x.device)
        with _on_device(x.device):
            _check(lib().heinsen_block_norms_backward(p, _ptr(d_r), _ptr(d_y), _ptr(dx), _ptr(dh), _ptr(dgate), _ptr(dpre),
                                                      _ptr(dpost), _ptr(ws), ws.numel(), _stream_ptr(x.device)))
        return dx, dh, dpre, dpost, dgate, None, None


def block_norms(x: torch.Tensor, branch: torch.Tensor, pre_weight: torch.Tensor, *, post_weight: torch.Tensor | None = None,
                gate: torch.Tensor | None = None, scale: float = 1.0, eps: float = 1e-6):
    """The norms before and after a block with its gate and residual scale; returns (r, y).  Asynchronous, differentiable.

    n = branch / sqrt(mean(branch^2) + eps) * post_weight (branch itself without post_weight); r = x + scale * gate * n;
    y = r / sqrt(mean(r^2) + eps) * pre_weight.  x, branch: contiguous [..., dim] of one dtype (float32 or bfloat16);
    gate: as x, or [..., 1, dim] for one gate per sequence; weights [dim], float32 or x's dtype.
    """
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, branch, pre_weight, post_weight, gate)):
        return _BlockNorms.apply(x, branch, pre_weight, post_weight, gate, float(scale), float(eps))
    p = _norms_problem("block_norms", x, pre_weight, float(eps), float(scale), branch, gate, post_weight)
    return _block_norms_forward(p, x)


class _GatedNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, weight, eps):
        p = _norms_problem("gated_norm", x, weight, eps, gate=gate)
        ctx.save_for_backward(x, gate, weight)
        ctx.eps = eps
        y = torch.empty_like(x)
        with _on_device(x.device):
            _check(lib().heinsen_gated_norm_forward(p, _ptr(y), _stream_ptr(x.device)))
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_y):
        x, gate, weight = ctx.saved_tensors
        p = _norms_problem("gated_norm", x, weight, ctx.eps, gate=gate)
        d_y = d_y.contiguous()
        dx, dweight = torch.empty_like(x), torch.empty_like(weight)
        dgate = None if gate is None else torch.empty_like(gate)
        ws = _space(int(lib().heinsen_gated_norm_workspace_bytes(p)), x.device)
        with _on_device(x.device):
            _check(lib().heinsen_gated_norm_backward(p, _ptr(d_y), _ptr(dx), _ptr(dgate), _ptr(dweight), _ptr(ws), ws.numel(),
                                                     _stream_ptr(x.device)))
        return dx, dgate, dweight, None


def gated_norm(x: torch.Tensor, gate: torch.Tensor | None, weight: torch.Tensor, *, eps: float = 1e-6) -> torch.Tensor:
    """x / sqrt(mean(x^2) + eps) * weight * silu(gate) over the last dimension (a head).  Asynchronous, differentiable.

    x, gate: contiguous [..., dim] of one dtype (float32 or bfloat16); gate None: no factor; weight [dim], float32 or x's."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, gate, weight)):
        return _GatedNorm.apply(x, gate, weight, float(eps))
    p = _norms_problem("gated_norm", x, weight, float(eps), gate=gate)
    y = torch.empty_like(x)
    with _on_device(x.device):
        _check(lib().heinsen_gated_norm_forward(p, _ptr(y), _stream_ptr(x.device)))
    return y
