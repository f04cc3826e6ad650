"""Python binding of include/heinsen_beam.h: beam search over models whose memory is a pool of states
(``heinsen_attention.decay_attention_step``, ``heinsen_delta.delta_attention_step``).

``beam_select`` picks the next beams from the logits of all of them, ``beam_reorder`` moves the states after their beams.  Every step
of the computation runs in the library's CUDA kernels; there is no CPU fallback.  Neither is differentiable.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from .heinsen_attention import _INT, _PTR, _SIZE, _I64, _addr, _cuda, _dtype, _dual_level, _increment_version, _launch, _no_tangents, _on_gpu, _space, _space_ok
from .heinsen_scan import lib as _scan_lib


class _Problem(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("vocabulary", ctypes.c_int64), ("beams", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("dtype", ctypes.c_int), ("logits", ctypes.c_void_p), ("batch_stride", ctypes.c_int64), ("beam_stride", ctypes.c_int64),
                ("scores", ctypes.c_void_p), ("ended", ctypes.c_void_p), ("end_token", ctypes.c_int64)]


_PROBLEM = struct.Struct("@qqiiiPqqPPq")
assert _PROBLEM.size == ctypes.sizeof(_Problem)

# Arguments and result of every function
_SIGNATURES = {
    "heinsen_beam_select": ([_Problem, _PTR, _PTR, _PTR, _PTR, _SIZE, _PTR], _INT),
    "heinsen_beam_workspace_bytes": ([_Problem], _SIZE),
    "heinsen_beam_reorder": ([_PTR, _I64, _I64, _PTR, _PTR, _I64, ctypes.c_int32, _PTR], _INT),
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
            return _bind(L["heinsen_beam_" + name], "heinsen_beam_" + name, lambda _: _PTR)

        self.select, self.space, self.reorder = of("select"), of("workspace_bytes"), of("reorder")


def _call() -> _Calls:
    global _calls
    if _calls is None:
        _calls = _Calls(lib())
    return _calls


def lib() -> ctypes.CDLL:
    """The shared library, with the functions of heinsen_beam.h bound.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = _scan_lib()
        for name in EXPORTS:
            _bind(getattr(L, name), name, ctypes.POINTER)
        _lib = L
    return _lib


def _select_problem(logits, scores, beams, ended, end_token) -> bytes:
    if logits.dim() != 3:
        raise ValueError("logits are [batch, beams, vocabulary]")
    b, w, n = logits.shape
    if scores.dtype is not torch.float32:
        raise TypeError("scores must be float32")
    if tuple(scores.shape) != (b, w) or not scores.is_contiguous():
        raise ValueError(f"scores must be contiguous, of shape {(b, w)}")
    sb, sw, sn = logits.stride()
    if sn != 1 and n > 1 and logits.numel():
        raise ValueError("logits: the last dimension must be contiguous")
    if ended is not None:
        if ended.dtype is not torch.bool and ended.dtype is not torch.uint8:
            raise TypeError("ended must be bool or uint8")
        if tuple(ended.shape) != (b, w) or not ended.is_contiguous():
            raise ValueError(f"ended must be contiguous, of shape {(b, w)}")
        if not 0 <= end_token < n:
            raise ValueError(f"end_token {end_token} is not one of {n} tokens")
    if not 1 <= w <= 64 or not 1 <= beams <= 64 or beams > w * n:
        raise ValueError(f"{beams} beams from {w} times {n} candidates: 1 to 64 of each, and no more than there are")
    _on_gpu(logits, "logits")
    _cuda("beam_select", logits.device, scores=scores, ended=ended)
    return _PROBLEM.pack(b, n, w, beams, _dtype(logits), logits.data_ptr(), sb, sw, scores.data_ptr(), 0 if ended is None else ended.data_ptr(),
                         end_token)


def workspace(logits: torch.Tensor, scores: torch.Tensor, beams: int | None = None) -> torch.Tensor:
    """Uninitialised scratch for ``beam_select`` calls of these shapes, one at a time."""
    return _space(_call().space(_select_problem(logits, scores, logits.shape[1] if beams is None else int(beams), None, 0)), logits.device)


def beam_select(logits: torch.Tensor, scores: torch.Tensor, beams: int | None = None, *, ended: torch.Tensor | None = None,
                end_token: int = 0, workspace: torch.Tensor | None = None):
    """The best continuations of each group of beams; returns (scores, parents, tokens), [B, beams] each.  Asynchronous.

    logits [B, W, N]: float32 or bfloat16, last dimension contiguous, any other strides; scores float32 [B, W]: the beams' log
    probabilities so far.  Of the W * N candidates scores[b, w] + log_softmax(logits[b, w])[n] the `beams` (default W) best are taken,
    best first, equal ones in the order of w * N + n (values count in 64 bits, and logits of one beam that even so have the same value
    stay in their order): their scores (float32), the beams w they continue and their tokens n (int32).
    ended [B, W] (bool or uint8): such a beam goes on with end_token alone, at its own score.  A beam that is not there has the score
    -inf; it, and one with a NaN or +inf among its logits, has candidates of -inf only, which come last.
    W and `beams` up to 64.  Logits are masked by -inf.  workspace: scratch from ``workspace()``, kept by the caller.
    """
    beams = logits.shape[1] if beams is None and logits.dim() == 3 else 0 if beams is None else int(beams)
    p = _select_problem(logits, scores, beams, ended, int(end_token))
    if _dual_level():
        _no_tangents("beam_select", logits, scores)
    dev = logits.device
    b = logits.shape[0]
    call = _call()
    if workspace is None:
        workspace = _space(call.space(p), dev)
    else:
        _space_ok(workspace, dev)
    values = torch.empty((b, beams), dtype=torch.float32, device=dev)
    chosen = torch.empty((2, b, beams), dtype=torch.int32, device=dev)
    parents, tokens = chosen.unbind(0)
    _launch(dev, call.select, p, values.data_ptr(), parents.data_ptr(), tokens.data_ptr(), workspace.data_ptr(), workspace.numel())
    return values, parents, tokens


def beam_reorder(state: torch.Tensor, parents: torch.Tensor, *, slots: torch.Tensor | None = None) -> torch.Tensor:
    """The states follow their beams, in place: beam w of group b has what beam parents[b, w] had.  Asynchronous; returns state.

    state [N, ...]: contiguous, any type, a pool of rows; parents int32 [B, W]; slots int32 [B, W]: the rows of the beams, or None for
    row b * W + w.  No two beams may share a row.  A beam with a parent outside of 0 .. W - 1, or with its own or its parent's slot
    outside of the pool, keeps what it has.  W up to 64.
    """
    if parents.dim() != 2 or parents.dtype is not torch.int32 or not parents.is_contiguous():
        raise ValueError("parents must be a contiguous int32 tensor [batch, beams]")
    b, w = parents.shape
    if slots is not None and (slots.dtype is not torch.int32 or slots.shape != parents.shape or not slots.is_contiguous()):
        raise ValueError("slots must be a contiguous int32 tensor [batch, beams]")
    if state.dim() < 1 or not state.is_contiguous():
        raise ValueError("state must be contiguous, [rows, ...]")
    if not 1 <= w <= 64:
        raise ValueError(f"{w} beams: 1 to 64 are possible")
    n = state.shape[0]
    if slots is None and n < b * w:
        raise ValueError(f"state has {n} rows for {b} times {w} beams")
    _on_gpu(state, "state")
    _cuda("beam_reorder", state.device, parents=parents, slots=slots)
    if _dual_level():
        _no_tangents("beam_reorder", state)
    row = state.numel() // n * state.element_size() if n else 0
    _launch(state.device, _call().reorder, state.data_ptr(), n, row, parents.data_ptr(), _addr(slots), b, w)
    _increment_version(state)
    return state
