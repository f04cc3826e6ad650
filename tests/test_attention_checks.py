"""Checks of arguments in the binding of heinsen_attention that need no GPU: what they refuse never reaches a kernel."""
import pytest
import torch


@pytest.fixture(scope="module")
def ha():
    from paper_2311_06281_b200 import build_ext, heinsen_attention
    build_ext.build()
    heinsen_attention.lib()
    return heinsen_attention


def test_a_kept_workspace_is_contiguous_bytes_of_the_calls_device(ha):
    gpu, host = torch.device("cuda", 0), torch.device("cpu")
    ws = torch.empty(512, dtype=torch.uint8)
    ha._space_ok(ws, host)
    with pytest.raises(ValueError, match="workspace is on cpu"):
        ha._space_ok(ws, gpu)
    with pytest.raises(ValueError, match="workspace is on meta"):
        ha._space_ok(torch.empty(512, dtype=torch.uint8, device="meta"), gpu)
    for bad in (ws.view(torch.float32), ws[::2], torch.empty(512, dtype=torch.int8)):
        with pytest.raises(ValueError, match="contiguous uint8"):
            ha._space_ok(bad, host)


def norms(ha, **other):
    d = dict(rows=6, gate_rows=3, dim=16, dtype=0, weight_dtype=0, scale=1.0, eps=1e-6, x=None, branch=None, gate=256, pre_weight=None,
             post_weight=None)
    d.update(other)
    return ha._Norms(*[d[n] for n, _ in ha._Norms._fields_])


def test_the_norms_scratch_is_zero_for_sizes_that_are_not_accepted(ha):
    """A gate of more rows than there are ended the process with a division by zero."""
    L = ha.lib()
    for space, own in ((L.heinsen_block_norms_workspace_bytes, [dict(gate_rows=12), dict(gate_rows=4), dict(gate_rows=0), dict(gate_rows=-3)]),
                       (L.heinsen_gated_norm_workspace_bytes, [])):
        assert space(norms(ha)) > 0 and space(norms(ha, rows=0)) > 0 and space(norms(ha, gate=None, gate_rows=12)) > 0
        for bad in (dict(rows=-1), dict(rows=1 << 62), dict(dim=0), dict(dim=16385), dict(dtype=7), dict(weight_dtype=1), dict(eps=-1.0), *own):
            assert space(norms(ha, **bad)) == 0, bad
        assert space(None) == 0


def test_strides_of_empty_tensors_are_not_looked_at(ha):
    """An expanded gradient without elements: PyTorch counts it as contiguous, so that no copy gives it other strides."""
    one = torch.zeros(())
    ha._rows(one.expand(0, 5, 2, 64).contiguous(), "d_o")
    ha._rows(one.expand(2, 3, 0, 16).contiguous(), "d_o")
    with pytest.raises(ValueError, match="contiguous"):
        ha._rows(one.expand(2, 3, 4, 16), "d_o")


def test_what_autograd_has_to_see(ha):
    from torch.autograd import forward_ad
    x, leaf = torch.ones(3), torch.ones(3, requires_grad=True)
    assert not ha._seen_by_autograd(x, None) and ha._seen_by_autograd(x, None, leaf)
    with torch.no_grad():
        assert not ha._seen_by_autograd(leaf)
    ha._no_tangents("a call", x)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, x)
        assert not dual.requires_grad and ha._seen_by_autograd(dual)
        ha._no_tangents("a call", x, leaf)
        with pytest.raises(NotImplementedError, match="a call"):
            ha._no_tangents("a call", x, dual)


def test_gradients_that_cannot_be_written_are_refused(ha):
    L = ha.lib()
    buf = torch.empty(1 << 16, dtype=torch.uint8)
    p = (buf.data_ptr() + 255) & ~255
    t = ha._Tensor(p, 64, 32, 16)

    def back(dq=p, dk=p, dv=p, d_state=None, scale=0.5, dtype=1):
        problem = ha._Problem(2, 4, 2, 2, 2, 2, 16, 16, dtype, scale, t, t, t, t, None, None)
        size = L.heinsen_attention_workspace_bytes(problem, 1)
        return L.heinsen_attention_backward(problem, t, d_state, dq, dk, dv, None, None, p, size, None)
    if not torch.cuda.is_available():  # what is accepted fails at the device
        assert back() in (2, 4) and back(d_state=p) in (2, 4) and back(dq=p + 4, dtype=0) in (2, 4) and back(scale=1e-39) in (2, 4)
    for bad in (dict(dq=p + 2), dict(dk=p + 8), dict(dv=p + 4), dict(scale=1e-39, d_state=p), dict(scale=-1e-40, d_state=p, dtype=0)):
        assert back(**bad) == 1, bad
