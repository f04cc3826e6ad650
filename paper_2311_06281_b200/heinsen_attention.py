"""Python binding of include/heinsen_attention.h: the recurrence with a matrix state (attention with a decay for each
head), its one-token step, and the norms around a block built on it.

    S_t = exp(log_a_t) S_{t-1} + k_t v_t^T,   o_t = scale * S_t^T q_t

As in ``heinsen_scan`` every step of the computation runs in the library's CUDA kernels; PyTorch provides device memory,
streams and the autograd graph.  There is no CPU fallback.  ``decay_attention``, ``block_norms`` and ``gated_norm`` are
differentiable in every tensor argument (once: their gradients are not differentiable again; backwards only: tangents of
``torch.autograd.forward_ad`` are refused).
"""
from __future__ import annotations

import ctypes
import struct

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version as _increment_version

from .heinsen_scan import HeinsenScanError, _check, _dtype_code, _on_device, lib as _scan_lib  # noqa: F401


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


_PROBLEM = struct.Struct("@qqiiiiiiif" + "Pqqq" * 4 + "PP")
_ROWS = struct.Struct("@Pqqq")
_NORMS = struct.Struct("@qqiiiffPPPPP0q")
assert (_PROBLEM.size, _ROWS.size, _NORMS.size) == tuple(ctypes.sizeof(t) for t in (_Problem, _Tensor, _Norms))

_lib = None
_calls = None

_PTR, _SIZE, _INT, _I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64
# Arguments (the problem first) and result of every function
_SIGNATURES = {
    "heinsen_attention_forward": ([_Problem, _Tensor, _PTR, _PTR, _SIZE, _PTR], _INT),
    "heinsen_attention_backward": ([_Problem, _Tensor, _PTR, _PTR, _PTR, _PTR, _PTR, _PTR, _PTR, _SIZE, _PTR], _INT),
    "heinsen_attention_workspace_bytes": ([_Problem, _INT], _SIZE),
    "heinsen_attention_step": ([_Problem, _Tensor, _PTR, _I64, _PTR, _PTR], _INT),
    "heinsen_attention_check": ([_PTR], _INT),
    "heinsen_block_norms_forward": ([_Norms, _PTR, _PTR, _PTR], _INT),
    "heinsen_block_norms_backward": ([_Norms, *[_PTR] * 8, _SIZE, _PTR], _INT),
    "heinsen_block_norms_workspace_bytes": ([_Norms], _SIZE),
    "heinsen_gated_norm_forward": ([_Norms, _PTR, _PTR], _INT),
    "heinsen_gated_norm_backward": ([_Norms, *[_PTR] * 5, _SIZE, _PTR], _INT),
    "heinsen_gated_norm_workspace_bytes": ([_Norms], _SIZE),
}
EXPORTS = list(_SIGNATURES)


def _bind(function, name: str, structure):
    """Gives a function its signature; `structure` maps a structure to the type that it is passed as."""
    args, function.restype = _SIGNATURES[name]
    function.argtypes = [structure(t) if issubclass(t, ctypes.Structure) else t for t in args]
    return function


class _Calls:
    """The functions once more, taking structures as packed bytes and pointers as integers: filling in ctypes structures
    field by field costs more than a small call does on the GPU."""

    def __init__(self, L):
        def of(name):
            return _bind(L[name], name, lambda _: _PTR)

        self.forward = of("heinsen_attention_forward")
        self.backward = of("heinsen_attention_backward")
        self.space = of("heinsen_attention_workspace_bytes")
        self.step = of("heinsen_attention_step")
        self.block_forward = of("heinsen_block_norms_forward")
        self.block_backward = of("heinsen_block_norms_backward")
        self.block_space = of("heinsen_block_norms_workspace_bytes")
        self.gated_forward = of("heinsen_gated_norm_forward")
        self.gated_backward = of("heinsen_gated_norm_backward")
        self.gated_space = of("heinsen_gated_norm_workspace_bytes")


def _call() -> _Calls:
    global _calls
    if _calls is None:
        _calls = _Calls(lib())
    return _calls


def lib() -> ctypes.CDLL:
    """The shared library, with the functions of heinsen_attention.h bound.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = _scan_lib()
        for name in EXPORTS:
            _bind(getattr(L, name), name, ctypes.POINTER)
        _lib = L
    return _lib


def _cuda(name: str, device, **tensors):
    for n, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name}: {n} is on {t.device}, not on {device}")


def _on_gpu(t: torch.Tensor, name: str):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (there is no CPU path)")


def _dtype(t: torch.Tensor) -> int:
    d = t.dtype
    return 1 if d is torch.bfloat16 else 0 if d is torch.float32 else _dtype_code(t)


def _addr(t):
    return None if t is None else t.data_ptr()


# The current stream's handle without an object around it: two microseconds of every call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _launch(device, fn, *args):
    """Calls fn(*args, stream) on `device` and its current stream."""
    index = device.index
    if index == torch.cuda.current_device():
        status = fn(*args, _raw_stream(index))
    else:
        with _on_device(device):
            status = fn(*args, _raw_stream(index))
    if status:
        _check(status)


def _seen_by_autograd(*tensors) -> bool:
    """Does a call have to go through its autograd function?  Where an input wants a gradient, and wherever tangents may be
    about (a dual tensor wants no gradient): the function refuses those."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                return True
    return _dual_level()


def _dual_level() -> bool:
    """May tensors have tangents at all?  (Asking each of them costs a microsecond.)"""
    return getattr(forward_ad, "_current_level", 0) >= 0


def _no_tangents(name, *tensors):
    if any(forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError(f"{name} has no forward-mode derivative")


def _space(nbytes: int, device) -> torch.Tensor:
    if nbytes == 0:
        raise ValueError("the library does not accept these sizes")
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


def _space_ok(workspace: torch.Tensor, device):
    """A caller's own scratch: the kernels are given its address."""
    if workspace.dtype is not torch.uint8 or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor")
    if workspace.device != device:
        raise ValueError(f"workspace is on {workspace.device}, not on {device}")


def _rows(t: torch.Tensor, name: str):
    """Address and strides of [batch, tokens, heads, dim], the last dimension contiguous."""
    s = t.stride()
    if s[3] != 1 and t.shape[3] > 1 and t.numel():  # an empty tensor counts as contiguous whatever its strides
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return t.data_ptr(), s[0], s[1], s[2]


def _state_ok(t, shape, name):
    if tuple(t.shape) != shape:
        raise ValueError(f"{name}: expected shape {shape}, got {tuple(t.shape)}")
    if t.dtype is not torch.float32:
        raise TypeError(f"{name} must be float32")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _heads(h, hq, hk, hv):
    if hq < 1 or hk < 1 or hv < 1 or h % hq or h % hk or h % hv:
        raise ValueError(f"the {h} heads of log_a must be a multiple of the heads of q ({hq}), k ({hk}) and v ({hv})")


class _Sizes:
    __slots__ = ("batch", "tokens", "heads", "k_dim", "v_dim", "packed")


def _problem(q, k, v, log_a, state0, scale, lengths) -> _Sizes:
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4:
        raise ValueError("q, k, v are [batch, tokens, heads, dim]")
    b, t, hq, kd = q.shape
    bk, tk, hk, kk = k.shape
    bv, tv, hv, vd = v.shape
    if bk != b or bv != b or tk != t or tv != t or kk != kd:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    if q.dtype is not k.dtype or q.dtype is not v.dtype:
        raise TypeError("q, k, v must share one dtype")
    if log_a.dtype is not torch.float32:
        raise TypeError("log_a must be float32")
    if log_a.dim() == 1:
        h, la = log_a.shape[0], (log_a.data_ptr(), 0, 0, log_a.stride(0))
    elif log_a.dim() == 3 and log_a.shape[:2] == (b, t):
        h, la = log_a.shape[2], (log_a.data_ptr(), *log_a.stride())
    else:
        raise ValueError(f"log_a: expected shape [heads] or {(b, t, 'heads')}, got {tuple(log_a.shape)}")
    _heads(h, hq, hk, hv)
    if state0 is not None:
        _state_ok(state0, (b, h, kd, vd), "state0")
    if lengths is not None and (lengths.dtype != torch.int32 or tuple(lengths.shape) != (b,) or not lengths.is_contiguous()):
        raise ValueError("lengths must be a contiguous int32 tensor [batch]")
    _on_gpu(q, "q")
    _cuda("decay_attention", q.device, k=k, v=v, log_a=log_a, state0=state0, lengths=lengths)
    p = _Sizes()
    p.batch, p.tokens, p.heads, p.k_dim, p.v_dim = b, t, h, kd, vd
    p.packed = _PROBLEM.pack(b, t, h, hq, hk, hv, kd, vd, _dtype(q), scale, *_rows(q, "q"), *_rows(k, "k"), *_rows(v, "v"), *la,
                             0 if state0 is None else state0.data_ptr(), 0 if lengths is None else lengths.data_ptr())
    return p


def _attention_forward(p: _Sizes, q: torch.Tensor, workspace: torch.Tensor | None):
    dev = q.device
    o = torch.empty((p.batch, p.tokens, p.heads, p.v_dim), dtype=q.dtype, device=dev)
    state = torch.empty((p.batch, p.heads, p.k_dim, p.v_dim), dtype=torch.float32, device=dev)
    call = _call()
    if workspace is None:
        workspace = _space(call.space(p.packed, 0), dev)
    else:
        _space_ok(workspace, dev)
    _launch(dev, call.forward, p.packed, _ROWS.pack(*_rows(o, "o")), state.data_ptr(), workspace.data_ptr(), workspace.numel())
    return o, state


class _DecayAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_a, state0, scale, lengths, workspace):
        o, state = _attention_forward(_problem(q, k, v, log_a, state0, scale, lengths), q, workspace)
        ctx.save_for_backward(q, k, v, log_a, state0, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, state

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_o, d_state):
        q, k, v, log_a, state0, lengths = ctx.saved_tensors
        dev = q.device
        need_decays = ctx.needs_input_grad[3]
        if need_decays and log_a.dim() == 3 and log_a.stride(0) == 0 and log_a.stride(1) == 0 and q.numel():
            log_a = log_a.contiguous()  # an expanded [heads]: its gradient is still asked for every token
        p = _problem(q, k, v, log_a, state0, ctx.scale, lengths)
        if d_o is None:
            d_o = torch.zeros((p.batch, p.tokens, p.heads, p.v_dim), dtype=q.dtype, device=dev)
        if d_o.shape[-1] > 1 and d_o.stride(-1) != 1:
            d_o = d_o.contiguous()
        if d_state is not None:
            d_state = d_state.contiguous()
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
        dla = torch.empty(log_a.shape, dtype=torch.float32, device=dev) if need_decays else None
        ds0 = torch.empty(state0.shape, dtype=torch.float32, device=dev) if ctx.needs_input_grad[4] else None
        call = _call()
        ws = _space(call.space(p.packed, 1), dev)
        _launch(dev, call.backward, p.packed, _ROWS.pack(*_rows(d_o, "d_o")), _addr(d_state), dq.data_ptr(), dk.data_ptr(),
                dv.data_ptr(), _addr(dla), _addr(ds0), ws.data_ptr(), ws.numel())
        return dq, dk, dv, dla, ds0, None, None, None


def workspace(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor) -> torch.Tensor:
    """Uninitialised scratch for ``decay_attention`` calls of these shapes, one at a time."""
    return _space(_call().space(_problem(q, k, v, log_a, None, 1.0, None).packed, 0), q.device)


def check(device) -> None:
    """Synchronises the current stream of `device` and raises if a bounded wait of any ``decay_attention`` call there, forward
    or backward, has run out on the device since the last check: the results of such a call are not valid."""
    device = torch.device(device)
    with _on_device(device):
        _check(lib().heinsen_attention_check(torch.cuda.current_stream(device).cuda_stream))


def decay_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor,
                    state0: torch.Tensor | None = None, *, scale: float | None = None,
                    lengths: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Attention with a decay for each head over whole sequences; returns (o, state).  Asynchronous, differentiable.

    q [B, T, Hq, K], k [B, T, Hk, K], v [B, T, Hv, V]: float32 or bfloat16, last dimension contiguous, any other strides;
    log_a: float32 [B, T, H], or [H] for fixed decays, H a multiple of Hq, Hk and Hv (head h reads head h * Hq // H of q);
    state0 [B, H, K, V] float32 continues earlier tokens; lengths [B] int32 ends row b after lengths[b] tokens.
    scale defaults to K ** -0.5.  o [B, T, H, V] has q's dtype, state [B, H, K, V] is float32 (what the next call or
    ``decay_attention_step`` takes).  log_a = -inf forgets the state at that token: packed sequences start so.  Log decays are
    meant to be <= 0.  A NaN or infinity in q, k or v spoils its row's heads from up to 127 tokens before it on.
    bfloat16 tensors (head dimensions in multiples of 8 to 128) go to the tensor cores, where the weights between tokens and the
    state that meets a query are rounded to bfloat16: results are 0.0023 off, of which 0.0017 are their own rounding; states and
    decay gradients are good to float32.  float32 tensors are computed in float32 throughout: cast to have that.
    workspace: scratch from ``workspace()``, kept by the caller; ``heinsen_scan.check(workspace)`` then reports what the
    device recorded for the last call (a bounded wait that ran out).  Without it each call takes its own; ``check(device)``
    reports for all calls, backward ones too.
    """
    scale = float(q.shape[-1] ** -0.5 if scale is None else scale)
    if _seen_by_autograd(q, k, v, log_a, state0):
        return _DecayAttention.apply(q, k, v, log_a, state0, scale, lengths, workspace)
    return _attention_forward(_problem(q, k, v, log_a, state0, scale, lengths), q, workspace)


def _step_problem(name, q, k, v, log_a, state, scale, slots, out):
    """The checks of a one-token call; returns the packed problem, the output, and what the call writes."""
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3:
        raise ValueError("q, k, v are [batch, heads, dim]")
    b, hq, kd = q.shape
    bk, hk, kk = k.shape
    bv, hv, vd = v.shape
    if bk != b or bv != b or kk != kd:
        raise ValueError(f"q {tuple(q.shape)}, k {tuple(k.shape)} and v {tuple(v.shape)} do not belong together")
    if q.dtype is not k.dtype or q.dtype is not v.dtype:
        raise TypeError("q, k, v must share one dtype")
    if log_a.dtype is not torch.float32:
        raise TypeError("log_a must be float32")
    if log_a.dim() == 1:
        h, ab, ah = log_a.shape[0], 0, log_a.stride(0)
    elif log_a.dim() == 2 and log_a.shape[0] == b:
        h, (ab, ah) = log_a.shape[1], log_a.stride()
    else:
        raise ValueError(f"log_a: expected shape [heads] or {(b, 'heads')}, got {tuple(log_a.shape)}")
    _heads(h, hq, hk, hv)
    n = state.shape[0]
    _state_ok(state, (n, h, kd, vd), "state")
    (qb, qh, q1), (kb, kh, k1), (vb, vh, v1) = q.stride(), k.stride(), v.stride()
    if b and ((q1 != 1 or k1 != 1) and kd > 1 or v1 != 1 and vd > 1):
        raise ValueError("q, k, v: the last dimension must be contiguous")
    if slots is None:
        if n < b:
            raise ValueError(f"state has {n} rows for {b} sequences")
    elif slots.dtype is not torch.int32 or tuple(slots.shape) != (b,) or not slots.is_contiguous():
        raise ValueError("slots must be a contiguous int32 tensor [batch]")
    dev = q.device
    _on_gpu(q, "q")
    written = state
    if out is None:
        out = torch.empty((b, h, vd), dtype=q.dtype, device=dev)
    elif tuple(out.shape) != (b, h, vd) or out.dtype is not q.dtype or b and out.stride(2) != 1 and vd > 1:
        raise ValueError("out must be [batch, heads, v_dim] of q's dtype, the last dimension contiguous")
    else:
        written = (state, out)
    _cuda(name, dev, k=k, v=v, log_a=log_a, state=state, slots=slots, out=out)
    packed = _PROBLEM.pack(b, 1, h, hq, hk, hv, kd, vd, _dtype(q), float(kd ** -0.5 if scale is None else scale),
                           q.data_ptr(), qb, 0, qh, k.data_ptr(), kb, 0, kh, v.data_ptr(), vb, 0, vh, log_a.data_ptr(), ab, 0, ah, 0, 0)
    return packed, out, written


def decay_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor, state: torch.Tensor, *,
                         scale: float | None = None, slots: torch.Tensor | None = None,
                         out: torch.Tensor | None = None) -> torch.Tensor:
    """One token for each sequence: updates ``state`` in place and returns o [B, H, V].  Asynchronous, not differentiable.

    q [B, Hq, K], k [B, Hk, K], v [B, Hv, V]; log_a float32 [B, H] or [H]; state float32 [N, H, K, V], of which sequence b
    uses row slots[b] (int32; negative or >= N: no state, o is zero), or row b.  No two sequences may share a row.
    """
    packed, out, written = _step_problem("decay_attention_step", q, k, v, log_a, state, scale, slots, out)
    if _dual_level():
        _no_tangents("decay_attention_step", q, k, v, log_a, state, out)
    ob, oh, _ = out.stride()
    _launch(q.device, _call().step, packed, _ROWS.pack(out.data_ptr(), ob, 0, oh), state.data_ptr(), state.shape[0], _addr(slots))
    # autograd sees no address being written to: a graph that kept what has been has to notice
    _increment_version(written)
    return out


# ------------------------------------------------------------------------------------------------------------- norms

def _norms_problem(name, x, weight, eps, scale=1.0, branch=None, gate=None, post=None) -> bytes:
    shape, dtype = x.shape, x.dtype
    dim = shape[-1]
    rows, gate_rows = x.numel() // dim if dim else 0, 1
    code = _dtype(x)
    if branch is not None and (branch.shape != shape or branch.dtype is not dtype):
        raise ValueError(f"{name}: branch must have the shape and dtype of x")
    if gate is not None:
        if gate.dtype is not dtype:
            raise TypeError(f"{name}: gate must have the dtype of x")
        if gate.shape != shape:
            # a gate for each sequence: [.., 1, dim] beside [.., tokens, dim]
            if branch is None or x.dim() < 2 or gate.shape != (*shape[:-2], 1, dim):
                raise ValueError(f"{name}: gate has shape {tuple(gate.shape)} beside {tuple(shape)}")
            gate_rows = max(1, shape[-2])
    for n, t in (("weight", weight), ("post_weight", post)):
        if t is not None and (t.dim() != 1 or t.shape[0] != dim):
            raise ValueError(f"{name}: {n} must be [{dim}]")
        if t is not None and t.dtype is not torch.float32 and t.dtype is not dtype:
            raise TypeError(f"{name}: {n} must be float32 or of x's dtype")
    if post is not None and post.dtype is not weight.dtype:
        raise TypeError(f"{name}: both weights must share one dtype")
    for n, t in (("x", x), ("branch", branch), ("gate", gate), ("weight", weight), ("post_weight", post)):
        if t is not None and not t.is_contiguous():
            raise ValueError(f"{name}: {n} must be contiguous")
    _on_gpu(x, "x")
    _cuda(name, x.device, branch=branch, gate=gate, weight=weight, post_weight=post)
    ptr = lambda t: t.data_ptr() if t is not None else 0  # noqa: E731
    return _NORMS.pack(rows, gate_rows, dim, code, _dtype(weight), scale, eps, x.data_ptr(), ptr(branch), ptr(gate), weight.data_ptr(),
                       ptr(post))


def _block_norms_forward(p: bytes, x):
    r, y = torch.empty_like(x), torch.empty_like(x)
    _launch(x.device, _call().block_forward, p, r.data_ptr(), y.data_ptr())
    return r, y


class _BlockNorms(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, branch, pre, post, gate, scale, eps):
        ctx.save_for_backward(x, branch, pre, post, gate)
        ctx.scale, ctx.eps = scale, eps
        ctx.set_materialize_grads(False)
        return _block_norms_forward(_norms_problem("block_norms", x, pre, eps, scale, branch, gate, post), x)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_r, d_y):
        x, branch, pre, post, gate = ctx.saved_tensors
        p = _norms_problem("block_norms", x, pre, ctx.eps, ctx.scale, branch, gate, post)  # a hook may have moved what was saved
        d_y = torch.zeros_like(x) if d_y is None else d_y.contiguous()
        d_r = None if d_r is None else d_r.contiguous()
        new = lambda t: None if t is None else torch.empty_like(t)  # noqa: E731
        dx, dh, dpre, dpost, dgate = new(x), new(branch), new(pre), new(post), new(gate)
        if dgate is not None and x.numel() == 0:
            dgate.zero_()  # gates of sequences without tokens: the library sees no rows, and so no gates
        call = _call()
        ws = _space(call.block_space(p), x.device)
        _launch(x.device, call.block_backward, p, _addr(d_r), d_y.data_ptr(), dx.data_ptr(), dh.data_ptr(), _addr(dgate),
                dpre.data_ptr(), _addr(dpost), ws.data_ptr(), ws.numel())
        return dx, dh, dpre, dpost, dgate, None, None


def block_norms(x: torch.Tensor, branch: torch.Tensor, pre_weight: torch.Tensor, *, post_weight: torch.Tensor | None = None,
                gate: torch.Tensor | None = None, scale: float = 1.0, eps: float = 1e-6):
    """The norms before and after a block with its gate and residual scale; returns (r, y).  Asynchronous, differentiable.

    n = branch / sqrt(mean(branch^2) + eps) * post_weight (branch itself without post_weight); r = x + scale * gate * n;
    y = r / sqrt(mean(r^2) + eps) * pre_weight.  x, branch: contiguous [..., dim] of one dtype (float32 or bfloat16);
    gate: as x, or [..., 1, dim] for one gate per sequence; weights [dim], float32 or x's dtype.
    """
    if _seen_by_autograd(x, branch, pre_weight, post_weight, gate):
        return _BlockNorms.apply(x, branch, pre_weight, post_weight, gate, float(scale), float(eps))
    return _block_norms_forward(_norms_problem("block_norms", x, pre_weight, float(eps), float(scale), branch, gate, post_weight), x)


class _GatedNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, weight, eps):
        ctx.save_for_backward(x, gate, weight)
        ctx.eps = eps
        y = torch.empty_like(x)
        _launch(x.device, _call().gated_forward, _norms_problem("gated_norm", x, weight, eps, gate=gate), y.data_ptr())
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_y):
        x, gate, weight = ctx.saved_tensors
        p = _norms_problem("gated_norm", x, weight, ctx.eps, gate=gate)  # a hook may have moved what was saved
        d_y = d_y.contiguous()
        dx, dweight = torch.empty_like(x), torch.empty_like(weight)
        dgate = None if gate is None else torch.empty_like(gate)
        call = _call()
        ws = _space(call.gated_space(p), x.device)
        _launch(x.device, call.gated_backward, p, d_y.data_ptr(), dx.data_ptr(), _addr(dgate), dweight.data_ptr(),
                ws.data_ptr(), ws.numel())
        return dx, dgate, dweight, None


def gated_norm(x: torch.Tensor, gate: torch.Tensor | None, weight: torch.Tensor, *, eps: float = 1e-6) -> torch.Tensor:
    """x / sqrt(mean(x^2) + eps) * weight * silu(gate) over the last dimension (a head).  Asynchronous, differentiable.

    x, gate: contiguous [..., dim] of one dtype (float32 or bfloat16); gate None: no factor; weight [dim], float32 or x's."""
    if _seen_by_autograd(x, gate, weight):
        return _GatedNorm.apply(x, gate, weight, float(eps))
    p = _norms_problem("gated_norm", x, weight, float(eps), gate=gate)
    y = torch.empty_like(x)
    _launch(x.device, _call().gated_forward, p, y.data_ptr())
    return y
