"""The functions of include/heinsen_delta.h and heinsen_beam.h are exported and bound, and refuse bad arguments before any CUDA
call.  No GPU needed."""
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, TOO_SMALL = 0, 1, 3


@pytest.fixture(scope="module")
def hd():
    from paper_2311_06281_b200 import build_ext, heinsen_delta
    build_ext.build()
    heinsen_delta.lib()
    return heinsen_delta


@pytest.fixture(scope="module")
def hb():
    from paper_2311_06281_b200 import build_ext, heinsen_beam
    build_ext.build()
    heinsen_beam.lib()
    return heinsen_beam


@pytest.fixture(scope="module")
def space():
    buf = np.zeros(1 << 16, dtype=np.float32)
    return buf, (buf.ctypes.data + 255) & ~255


@pytest.mark.parametrize("name", ["delta", "beam"])
def test_every_declared_function_is_exported_and_bound(hd, hb, name):
    text = open(os.path.join(ROOT, "include", f"heinsen_{name}.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(heinsen_\w+)\s*\(", text)))
    m = {"delta": hd, "beam": hb}[name]
    assert names == sorted(m.EXPORTS)
    for n in names:
        assert getattr(m.lib(), n).argtypes is not None


def delta_problem(hd, p, beta=True, **other):
    from paper_2311_06281_b200 import heinsen_attention as ha
    t = ha._Tensor(p, 64, 32, 16)
    d = dict(batch=2, tokens=4, heads=4, q_heads=4, k_heads=2, v_heads=1, k_dim=16, v_dim=8, dtype=0, scale=0.5, q=t, k=t, v=t,
             log_a=t, state0=None, lengths=None)
    d.update(other)
    return hd._Delta(ha._Problem(*[d[n] for n, _ in ha._Problem._fields_]), t if beta else ha._Tensor(None, 1, 1, 1))


def test_delta_arguments_are_checked_on_the_host(hd, space):
    from paper_2311_06281_b200 import heinsen_attention as ha
    L, (_, p) = hd.lib(), space
    o = ha._Tensor(p, 64, 32, 16)
    forward = lambda pr, ws=p, size=1 << 30, out=o: L.heinsen_delta_forward(pr, out, None, ws, size, None)  # noqa: E731
    backward = lambda pr, ws=p, size=1 << 40, g=o, dq=p: L.heinsen_delta_backward(pr, g, None, dq, p, p, None, None, None, ws, size, None)  # noqa: E731
    assert forward(delta_problem(hd, p, batch=0)) == OK and forward(delta_problem(hd, p, heads=0)) == OK
    for bad in (dict(batch=-1), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=-4), dict(q_heads=3), dict(k_heads=0), dict(v_heads=8),
                dict(k_dim=0), dict(k_dim=257), dict(v_dim=257), dict(dtype=2), dict(scale=0.0), dict(scale=float("nan")), dict(batch=1 << 30)):
        assert forward(delta_problem(hd, p, **bad)) == INVALID and backward(delta_problem(hd, p, **bad)) == INVALID, bad
        assert L.heinsen_delta_workspace_bytes(delta_problem(hd, p, **bad), 0) == L.heinsen_delta_workspace_bytes(delta_problem(hd, p, **bad), 1) == 0
    for name in ("q", "k", "v", "log_a"):
        bad = delta_problem(hd, p, **{name: ha._Tensor(None, 1, 1, 1)})
        assert forward(bad) == INVALID and backward(bad) == INVALID, name
    good = delta_problem(hd, p)
    assert forward(delta_problem(hd, p, beta=False)) == INVALID and backward(delta_problem(hd, p, beta=False)) == INVALID
    for call in (forward, backward):
        assert call(None) == INVALID and call(good, None) == INVALID and call(good, p + 8) == INVALID and call(good, p, 16) == TOO_SMALL
    assert forward(good, out=None) == INVALID and backward(good, g=None) == INVALID and backward(good, dq=None) == INVALID
    assert L.heinsen_delta_workspace_bytes(None, 0) == 0
    # tensors that TMA loads as they are need no copy; of the forward call only the chunks' images remain
    aligned = dict(dtype=1, k_dim=16, v_dim=16, q=ha._Tensor(p, 64, 32, 16), k=ha._Tensor(p, 64, 32, 16), v=ha._Tensor(p, 64, 32, 16))
    plain = L.heinsen_delta_workspace_bytes(delta_problem(hd, p, **aligned), 0)
    shifted = L.heinsen_delta_workspace_bytes(delta_problem(hd, p, **{**aligned, "v": ha._Tensor(p + 2, 64, 32, 16)}), 0)
    assert 0 < plain < shifted


def test_delta_step_arguments(hd, space):
    from paper_2311_06281_b200 import heinsen_attention as ha
    L, (_, p) = hd.lib(), space
    o = ha._Tensor(p, 64, 32, 16)
    step = lambda pr, pool=4, slots=None, out=o, state=p: L.heinsen_delta_step(pr, out, state, pool, slots, None)  # noqa: E731
    one = lambda **k: delta_problem(hd, p, **{"tokens": 1, **k})  # noqa: E731
    assert step(one(batch=0)) == OK
    for bad in (one(tokens=2), one(state0=p), one(lengths=p), one(k_dim=300), one(q=ha._Tensor(None, 1, 1, 1)), one(beta=False)):
        assert step(bad) == INVALID
    assert step(one(), pool=1) == INVALID and step(one(), pool=-1) == INVALID and step(one(), out=None) == INVALID and step(one(), state=None) == INVALID


def test_the_delta_binding_refuses(hd):
    f = lambda *s, **k: torch.zeros(*s, **k)  # noqa: E731
    q, la, beta = f(2, 5, 4, 16), f(2, 5, 4), f(2, 5, 4)
    for call, error, text in (
            (lambda: hd.delta_attention(q, q, q, la, beta), ValueError, "CUDA"),
            (lambda: hd.delta_attention(q[0], q, q, la, beta), ValueError, "tokens, heads, dim"),
            (lambda: hd.delta_attention(q, q[:, :4], q, la, beta), ValueError, "belong together"),
            (lambda: hd.delta_attention(q, q, q.bfloat16(), la, beta), TypeError, "one dtype"),
            (lambda: hd.delta_attention(q, q, q, la.double(), beta), TypeError, "log_a must be float32"),
            (lambda: hd.delta_attention(q, q, q, la[:, :4], beta), ValueError, "log_a"),
            (lambda: hd.delta_attention_step(q[:, 0], q[:, 0], q[:, 0], la[:, 0], beta[:, 0], f(1, 4, 16, 16)), ValueError, "1 rows for 2"),
            (lambda: hd.delta_attention_step(q[:, 0], q[:, 0], q[:, 0], la[:, 0], beta[:, 0], f(2, 4, 16, 16).double()), TypeError, "float32"),
            (lambda: hd.delta_attention_step(q[:, 0], q[:, 0], q[:, 0], la[:, 0], beta[:, 0], f(2, 4, 16, 16)), ValueError, "CUDA")):
        with pytest.raises(error, match=text):
            call()
    cpu = torch.device("cpu")
    hd._beta_ok(beta, (2, 5, 4), cpu)
    with pytest.raises(TypeError, match="beta must be float32"):
        hd._beta_ok(beta.bfloat16(), (2, 5, 4), cpu)
    with pytest.raises(ValueError, match="beta: expected shape"):
        hd._beta_ok(beta[0], (2, 5, 4), cpu)
    with pytest.raises(ValueError, match="beta is on cpu"):
        hd._beta_ok(beta, (2, 5, 4), torch.device("cuda", 0))


def beam_problem(hb, p, **other):
    d = dict(batch=2, vocabulary=50, beams=3, keep=4, dtype=0, logits=p, batch_stride=150, beam_stride=50, scores=p, ended=None, end_token=0)
    d.update(other)
    return hb._Problem(*[d[n] for n, _ in hb._Problem._fields_])


def test_beam_arguments_are_checked_on_the_host(hb, space):
    L, (_, p) = hb.lib(), space
    select = lambda pr, ws=p, size=1 << 20, out=p: L.heinsen_beam_select(pr, out, p, p, ws, size, None)  # noqa: E731
    assert select(beam_problem(hb, p, batch=0)) == OK
    for bad in (dict(batch=-1), dict(vocabulary=0), dict(vocabulary=1 << 31), dict(beams=0), dict(beams=65), dict(keep=0), dict(keep=65),
                dict(vocabulary=1, keep=4), dict(dtype=2), dict(ended=p, end_token=-1), dict(ended=p, end_token=50), dict(batch=1 << 30)):
        assert select(beam_problem(hb, p, **bad)) == INVALID, bad
        assert L.heinsen_beam_workspace_bytes(beam_problem(hb, p, **bad)) == 0, bad
    for bad in (dict(logits=None), dict(scores=None), dict(logits=p + 2)):
        assert select(beam_problem(hb, p, **bad)) == INVALID, bad
    good = beam_problem(hb, p)
    assert select(None) == INVALID and select(good, None) == INVALID and select(good, p + 8) == INVALID and select(good, p, 16) == TOO_SMALL
    assert select(good, out=None) == INVALID
    reorder = lambda state=p, pool=8, row=16, parents=p, slots=None, batch=2, beams=3: L.heinsen_beam_reorder(state, pool, row, parents, slots, batch, beams, None)  # noqa: E731
    assert reorder(batch=0) == OK and reorder(pool=0, slots=p) == OK and reorder(row=0) == OK
    for bad in (dict(pool=-1), dict(row=-1), dict(batch=-1), dict(beams=0), dict(beams=65), dict(pool=5), dict(state=None), dict(parents=None),
                dict(pool=1 << 40, row=1 << 40), dict(batch=1 << 30)):
        assert reorder(**bad) == INVALID, bad


def test_the_beam_binding_refuses(hb):
    f = lambda *s, **k: torch.zeros(*s, **k)  # noqa: E731
    logits, scores, i32 = f(2, 3, 10), f(2, 3), dict(dtype=torch.int32)
    for call, error, text in (
            (lambda: hb.beam_select(logits, scores), ValueError, "CUDA"),
            (lambda: hb.beam_select(logits[0], scores, 2), ValueError, "batch, beams, vocabulary"),
            (lambda: hb.beam_select(logits[0], scores), ValueError, "batch, beams, vocabulary"),
            (lambda: hb.beam_select(logits, scores.double()), TypeError, "float32"),
            (lambda: hb.beam_select(logits, scores[:1]), ValueError, "scores"),
            (lambda: hb.beam_select(logits, f(3, 2).T), ValueError, "contiguous"),
            (lambda: hb.beam_select(logits.transpose(1, 2), f(2, 10)), ValueError, "last dimension"),
            (lambda: hb.beam_select(logits, scores, 31), ValueError, "candidates"),
            (lambda: hb.beam_select(logits, scores, 0), ValueError, "candidates"),
            (lambda: hb.beam_select(f(1, 65, 10), f(1, 65), 4), ValueError, "candidates"),
            (lambda: hb.beam_select(logits, scores, ended=f(2, 3)), TypeError, "bool"),
            (lambda: hb.beam_select(logits, scores, ended=f(2, 2, dtype=torch.bool)), ValueError, "ended"),
            (lambda: hb.beam_select(logits, scores, ended=f(2, 3, dtype=torch.bool), end_token=10), ValueError, "end_token"),
            (lambda: hb.beam_reorder(f(6, 4), f(2, 3, **i32)), ValueError, "CUDA"),
            (lambda: hb.beam_reorder(f(5, 4), f(2, 3, **i32)), ValueError, "5 rows"),
            (lambda: hb.beam_reorder(f(6, 4), f(2, 3, dtype=torch.int64)), ValueError, "parents"),
            (lambda: hb.beam_reorder(f(6, 4), f(2, 3, **i32), slots=f(3, 2, **i32)), ValueError, "slots"),
            (lambda: hb.beam_reorder(f(4, 6).T, f(2, 3, **i32)), ValueError, "contiguous"),
            (lambda: hb.beam_reorder(f(200, 6), f(2, 65, **i32)), ValueError, "65 beams")):
        with pytest.raises(error, match=text):
            call()
