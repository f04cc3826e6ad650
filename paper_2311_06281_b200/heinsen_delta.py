"""Python binding of include/heinsen_delta.h: the delta rule with a decay for each head, and its one-token step.

    S_t = exp(log_a_t) S_{t-1} + beta_t k_t (v_t - exp(log_a_t) S_{t-1}^T k_t)^T,   o_t = scale * S_t^T q_t

The recurrence of ``heinsen_attention.decay_attention`` with a write that first takes out what the state already answers for
the key.  As there every step of the computation runs in the library's CUDA kernels, there is no CPU fallback, and
``delta_attention`` is differentiable in every tensor argument (once, backwards only).
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import heinsen_attention as _ha
from .heinsen_attention import _INT, _PROBLEM, _PTR, _ROWS, _SIZE, _I64, _Problem, _Tensor, _addr, _cuda, _launch, _rows, _space, _space_ok
from .heinsen_scan import _check, _on_device, lib as _scan_lib


class _Delta(ctypes.Structure):
    _fields_ = [("a", _Problem), ("beta", _Tensor)]


_DELTA = struct.Struct(_PROBLEM.format + "Pqqq")
assert _DELTA.size == ctypes.sizeof(_Delta)

# Arguments (the problem first) and result of every function
_SIGNATURES = {
    "heinsen_delta_forward": ([_Delta, _Tensor, _PTR, _PTR, _SIZE, _PTR], _INT),
    "heinsen_delta_backward": ([_Delta, _Tensor, _PTR, _PTR, _PTR, _PTR, _PTR, _PTR, _PTR, _PTR, _SIZE, _PTR], _INT),
    "heinsen_delta_workspace_bytes": ([_Delta, _INT], _SIZE),
    "heinsen_delta_step": ([_Delta, _Tensor, _PTR, _I64, _PTR, _PTR], _INT),
    "heinsen_delta_check": ([_PTR], _INT),
}
EXPORTS = list(_SIGNATURES)

_lib = None
_calls = None


def _bind(function, name: str, structure):
    args, function.restype = _SIGNATURES[name]
    function.argtypes = [structure(t) if issubclass(t, ctypes.Structure) else t for t in args]
    return function


class _Calls:
    """The functions once more, taking structures as packed bytes and pointers as integers."""

    def __init__(self, L):
        def of(name):
            return _bind(L["heinsen_delta_" + name], "heinsen_delta_" + name, lambda _: _PTR)

        self.forward, self.backward, self.space, self.step = of("forward"), of("backward"), of("workspace_bytes"), of("step")


def _call() -> _Calls:
    global _calls
    if _calls is None:
        _calls = _Calls(lib())
    return _calls


def lib() -> ctypes.CDLL:
    """The shared library, with the functions of heinsen_delta.h bound.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = _scan_lib()
        for name in EXPORTS:
            _bind(getattr(L, name), name, ctypes.POINTER)
        _lib = L
    return _lib


def _beta_ok(beta, shape, device):
    if beta.dtype is not torch.float32:
        raise TypeError("beta must be float32")
    if tuple(beta.shape) != shape:
        raise ValueError(f"beta: expected shape {shape}, got {tuple(beta.shape)}")
    _cuda("delta_attention", device, beta=beta)


def _problem(q, k, v, log_a, beta, state0, scale, lengths) -> _ha._Sizes:
    p = _ha._problem(q, k, v, log_a, state0, scale, lengths)
    _beta_ok(beta, (p.batch, p.tokens, p.heads), q.device)
    p.packed += struct.pack("@Pqqq", beta.data_ptr(), *beta.stride())
    return p


def _forward(p: _ha._Sizes, q: torch.Tensor, workspace: torch.Tensor | None):
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


class _DeltaAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_a, beta, state0, scale, lengths, workspace):
        o, state = _forward(_problem(q, k, v, log_a, beta, state0, scale, lengths), q, workspace)
        ctx.save_for_backward(q, k, v, log_a, beta, state0, lengths)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, state

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, d_o, d_state):
        q, k, v, log_a, beta, state0, lengths = ctx.saved_tensors
        dev = q.device
        need_decays, need_beta = ctx.needs_input_grad[3], ctx.needs_input_grad[4]
        if need_decays and log_a.dim() == 3 and log_a.stride(0) == 0 and log_a.stride(1) == 0 and q.numel():
            log_a = log_a.contiguous()  # an expanded [heads]: its gradient is still asked for every token
        p = _problem(q, k, v, log_a, beta, state0, ctx.scale, lengths)
        if d_o is None:
            d_o = torch.zeros((p.batch, p.tokens, p.heads, p.v_dim), dtype=q.dtype, device=dev)
        if d_o.shape[-1] > 1 and d_o.stride(-1) != 1:
            d_o = d_o.contiguous()
        if d_state is not None:
            d_state = d_state.contiguous()
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
        dla = torch.empty(log_a.shape, dtype=torch.float32, device=dev) if need_decays else None
        dbeta = torch.empty(beta.shape, dtype=torch.float32, device=dev) if need_beta else None
        ds0 = torch.empty(state0.shape, dtype=torch.float32, device=dev) if ctx.needs_input_grad[5] else None
        call = _call()
        ws = _space(call.space(p.packed, 1), dev)
        _launch(dev, call.backward, p.packed, _ROWS.pack(*_rows(d_o, "d_o")), _addr(d_state), dq.data_ptr(), dk.data_ptr(),
                dv.data_ptr(), _addr(dla), _addr(dbeta), _addr(ds0), ws.data_ptr(), ws.numel())
        return dq, dk, dv, dla, dbeta, ds0, None, None, None


def workspace(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor, beta: torch.Tensor) -> torch.Tensor:
    """Uninitialised scratch for ``delta_attention`` calls of these shapes, strides and alignments, one at a time."""
    return _space(_call().space(_problem(q, k, v, log_a, beta, None, 1.0, None).packed, 0), q.device)


def check(device) -> None:
    """Synchronises the current stream of `device` and raises if a bounded wait of any ``delta_attention`` call there, forward
    or backward, has run out on the device since the last check: the results of such a call are not valid."""
    device = torch.device(device)
    with _on_device(device):
        _check(lib().heinsen_delta_check(torch.cuda.current_stream(device).cuda_stream))


def delta_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor, beta: torch.Tensor,
                    state0: torch.Tensor | None = None, *, scale: float | None = None, lengths: torch.Tensor | None = None,
                    workspace: torch.Tensor | None = None):
    """The delta rule with a decay over whole sequences; returns (o, state).  Asynchronous, differentiable.

    q [B, T, Hq, K], k [B, T, Hk, K], v [B, T, Hv, V]: float32 or bfloat16, last dimension contiguous, any other strides;
    log_a: float32 [B, T, H], or [H] for fixed decays (zeros: none), H a multiple of Hq, Hk and Hv (head h reads head
    h * Hq // H of q); beta: float32 [B, T, H], the share of the error that is written, 0 to 1 (or 2) for keys of length one;
    keys are taken as they are.  state0 [B, H, K, V] float32 continues earlier tokens; lengths [B] int32 ends row b after
    lengths[b] tokens.  scale defaults to K ** -0.5.  o [B, T, H, V] has q's dtype, state [B, H, K, V] is float32 (what the next
    call or ``delta_attention_step`` takes).  log_a = -inf forgets the state, whatever it holds, at that token: packed sequences start so.
    A NaN or infinity in q, k or v spoils its row's heads from up to 63 tokens before it on.
    The products run on the tensor cores.  float32 tensors count with 24 bits.  Of bfloat16 tensors the state and the gradients
    of log_a, beta and state0 do too (1e-7 to 8e-7 off); what o, dq and dk are products with counts with 16, so that they are off by
    their own rounding to bfloat16 alone (1.7e-3 in the mean).
    workspace: scratch from ``workspace()``, kept by the caller; ``heinsen_scan.check(workspace)`` then reports what the
    device recorded for the last call (a bounded wait that ran out).  Without it each call takes its own; ``check(device)``
    reports for all calls, backward ones too.
    """
    scale = float(q.shape[-1] ** -0.5 if scale is None else scale)
    if _ha._seen_by_autograd(q, k, v, log_a, beta, state0):
        return _DeltaAttention.apply(q, k, v, log_a, beta, state0, scale, lengths, workspace)
    return _forward(_problem(q, k, v, log_a, beta, state0, scale, lengths), q, workspace)


def delta_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, log_a: torch.Tensor, beta: torch.Tensor,
                         state: torch.Tensor, *, scale: float | None = None, slots: torch.Tensor | None = None,
                         out: torch.Tensor | None = None) -> torch.Tensor:
    """One token for each sequence: updates ``state`` in place and returns o [B, H, V].  Asynchronous, not differentiable.

    q [B, Hq, K], k [B, Hk, K], v [B, Hv, V]; log_a float32 [B, H] or [H]; beta float32 [B, H]; state float32 [N, H, K, V], of
    which sequence b uses row slots[b] (int32; negative or >= N: no state, o is zero), or row b.  No two sequences may share a row.
    """
    packed, out, written = _ha._step_problem("delta_attention_step", q, k, v, log_a, state, scale, slots, out)
    _beta_ok(beta, (q.shape[0], log_a.shape[-1]), q.device)
    if _ha._dual_level():
        _ha._no_tangents("delta_attention_step", q, k, v, log_a, beta, state, out)
    bb, bh = beta.stride()
    ob, oh, _ = out.stride()
    _launch(q.device, _call().step, packed + struct.pack("@Pqqq", beta.data_ptr(), bb, 0, bh), _ROWS.pack(out.data_ptr(), ob, 0, oh),
            state.data_ptr(), state.shape[0], _addr(slots))
    _ha._increment_version(written)
    return out
