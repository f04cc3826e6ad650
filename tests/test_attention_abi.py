"""The functions of include/heinsen_attention.h are exported and bound, and refuse bad arguments before any CUDA call.
No GPU needed."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, TOO_SMALL = 0, 1, 3


@pytest.fixture(scope="module")
def ha():
    from paper_2311_06281_b200 import build_ext, heinsen_attention
    build_ext.build()
    heinsen_attention.lib()
    return heinsen_attention


def test_every_declared_function_is_exported_and_bound(ha):
    text = open(os.path.join(ROOT, "include", "heinsen_attention.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(heinsen_\w+)\s*\(", text)))
    assert names == sorted(ha.EXPORTS)
    for n in names:
        assert getattr(ha.lib(), n).argtypes is not None


def problem(ha, p, **other):
    t = ha._Tensor(p, 64, 32, 16)
    d = dict(batch=2, tokens=4, heads=4, q_heads=4, k_heads=2, v_heads=1, k_dim=16, v_dim=8, dtype=0, scale=0.5, q=t, k=t, v=t,
             log_a=t, state0=None, lengths=None)
    d.update(other)
    return ha._Problem(*[d[n] for n, _ in ha._Problem._fields_])


def test_attention_arguments_are_checked_on_the_host(ha):
    L = ha.lib()
    buf = np.zeros(4096, dtype=np.float32)
    p = (buf.ctypes.data + 255) & ~255
    o = ha._Tensor(p, 64, 32, 16)
    forward = lambda pr, ws=p, size=1 << 20: L.heinsen_attention_forward(pr, o, None, ws, size, None)  # noqa: E731
    # nothing to do
    assert forward(problem(ha, p, batch=0)) == OK and forward(problem(ha, p, heads=0)) == OK
    for bad in (dict(batch=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=-4), dict(q_heads=3), dict(k_heads=0),
                dict(v_heads=8), dict(k_dim=0), dict(k_dim=257), dict(v_dim=257), dict(dtype=2), dict(scale=0.0),
                dict(scale=float("nan")), dict(batch=1 << 30)):
        assert forward(problem(ha, p, **bad)) == INVALID, bad
        assert L.heinsen_attention_workspace_bytes(problem(ha, p, **bad), 1) == 0, bad
    for name in ("q", "k", "v", "log_a"):
        assert forward(problem(ha, p, **{name: ha._Tensor(None, 1, 1, 1)})) == INVALID, name
    assert forward(problem(ha, p), None) == INVALID and forward(problem(ha, p), p + 8) == INVALID
    assert forward(problem(ha, p), p, 16) == TOO_SMALL
    assert forward(None) == INVALID
    assert L.heinsen_attention_forward(problem(ha, p), None, None, p, 1 << 20, None) == INVALID
    size = L.heinsen_attention_workspace_bytes(problem(ha, p), 1)
    assert size >= 2 * 4 * 4 * (16 + 16 + 8) * 4
    back = lambda **o2: L.heinsen_attention_backward(  # noqa: E731
        problem(ha, p), o2.get("d_o", o), None, o2.get("dq", p), p, p, None, None, p, o2.get("size", size), None)
    assert back(d_o=ha._Tensor(None, 1, 1, 1)) == INVALID and back(dq=None) == INVALID and back(size=size - 1) == TOO_SMALL
    step = lambda pr, pool, n: L.heinsen_attention_step(pr, o, pool, n, None, None)  # noqa: E731
    one = problem(ha, p, tokens=1)
    assert step(problem(ha, p), p, 2) == INVALID                       # more than one token
    assert step(one, p, 1) == INVALID and step(one, p, -1) == INVALID    # fewer states than sequences
    assert step(one, None, 2) == INVALID
    assert step(problem(ha, p, tokens=1, lengths=p), p, 2) == INVALID
    assert step(problem(ha, p, tokens=1, batch=0), None, 0) == OK


def test_norm_arguments_are_checked_on_the_host(ha):
    L = ha.lib()
    buf = np.zeros(4096, dtype=np.float32)
    p = (buf.ctypes.data + 255) & ~255

    def norms(**other):
        d = dict(rows=6, gate_rows=3, dim=16, dtype=0, weight_dtype=0, scale=1.0, eps=1e-6, x=p, branch=p, gate=p, pre_weight=p,
                 post_weight=p)
        d.update(other)
        return ha._Norms(*[d[n] for n, _ in ha._Norms._fields_])

    assert L.heinsen_block_norms_forward(norms(rows=0), p, p, None) == OK and L.heinsen_gated_norm_forward(norms(rows=0), p, None) == OK
    for bad in (dict(rows=-1), dict(dim=0), dict(dim=16385), dict(dtype=5), dict(weight_dtype=1), dict(eps=-1.0),
                dict(eps=float("nan")), dict(scale=float("inf")), dict(gate_rows=4), dict(gate_rows=0), dict(x=None),
                dict(branch=None), dict(pre_weight=None)):
        assert L.heinsen_block_norms_forward(norms(**bad), p, p, None) == INVALID, bad
    assert L.heinsen_block_norms_forward(norms(), None, p, None) == INVALID
    assert L.heinsen_gated_norm_forward(norms(), None, None) == INVALID
    size = L.heinsen_block_norms_workspace_bytes(norms())
    assert size > 0
    assert L.heinsen_block_norms_backward(norms(), None, p, p, p, p, p, p, p, size - 1, None) == TOO_SMALL
    assert L.heinsen_block_norms_backward(norms(), None, p, p, p, None, p, p, p, size, None) == INVALID   # a gate without dgate
    assert L.heinsen_block_norms_backward(norms(), None, None, p, p, p, p, p, p, size, None) == INVALID
    assert L.heinsen_gated_norm_backward(norms(), p, p, p, None, p, size, None) == INVALID


def test_without_a_gpu_the_calls_fail_loudly(ha):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    q, a, s = torch.zeros(1, 2, 1, 8), torch.zeros(1, 2, 1), torch.zeros(1, 1, 8, 8)
    for call in (lambda: ha.decay_attention(q, q, q, a), lambda: ha.decay_attention_step(q[:, 0], q[:, 0], q[:, 0], a[:, 0], s),
                 lambda: ha.block_norms(q, q, torch.ones(8)), lambda: ha.gated_norm(q, q, torch.ones(8))):
        with pytest.raises(ValueError):
            call()
    buf = ctypes.create_string_buffer(8192)
    p = (ctypes.addressof(buf) + 255) & ~255
    assert ha.lib().heinsen_attention_forward(problem(ha, p), ha._Tensor(p, 64, 32, 16), None, p, 4096, None) in (2, 4)
