"""The attention with a decay for each head where sequences are cut into segments (few heads, many tokens): outputs, states and
every gradient, with ends, resets and empty rows inside, at and behind the cuts; tolerances as in attention_testlib."""
import pytest
import torch

from attention_testlib import attention64, close, leaf64
from test_gpu_attention import BF16, DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu

# (b, t, h, hq, hk, hv, kd, vd), dtype, lengths: bf16 is cut at multiples of 128 tokens, float32 and odd widths at those of 32
CASES = [
    ((1, 1500, 2, 2, 2, 2, 64, 128), BF16, None),
    ((1, 1536, 1, 1, 1, 1, 128, 128), BF16, None),
    ((3, 1300, 2, 2, 1, 2, 128, 72), BF16, (1300, 0, 140)),
    ((2, 1281, 3, 1, 3, 1, 96, 64), BF16, (1, 1280)),
    ((1, 200, 2, 2, 2, 2, 64, 64), F32, None),
    ((3, 161, 4, 4, 2, 1, 33, 65), F32, (161, 0, 33)),
    ((2, 128, 1, 1, 1, 1, 256, 20), F32, (32, 127)),
    ((1, 400, 2, 1, 2, 2, 128, 256), F32, None),
    ((2, 300, 2, 2, 2, 2, 50, 7), BF16, (300, 65)),
]


def inputs(shape, dtype, lengths, decay, seed):
    q, k, v, log_a, s0 = make(*shape, dtype, decay, True, seed=seed)
    ends = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    if lengths is not None:  # what lies behind the ends is not read
        behind = torch.arange(shape[1], device=DEV)[None] >= ends[:, None]
        q, k, v = (x.masked_fill(behind[..., None, None], float("nan")) for x in (q, k, v))
        if log_a.dim() == 3:
            log_a = log_a.masked_fill(behind[..., None], float("nan"))
    return q, k, v, log_a, s0, ends


def clean(*tensors):
    return [torch.nan_to_num(x, nan=0.0, neginf=-float("inf"), posinf=float("inf")) for x in tensors]


@pytest.mark.parametrize("decay", ["token", "head", "strong", "reset"])
@pytest.mark.parametrize("shape,dtype,lengths", CASES, ids=str)
def test_forward_over_cuts(ha, shape, dtype, lengths, decay):  # noqa: F811
    q, k, v, log_a, s0, ends = inputs(shape, dtype, lengths, decay, 11 + sum(shape))
    o, s = ha.decay_attention(q, k, v, log_a, s0, lengths=ends)
    want_o, want_s = attention64(*clean(q, k, v, log_a), s0, shape[6] ** -0.5, ends)
    close(o, want_o, "o")
    close(s, want_s, "state")
    again_o, again_s = ha.decay_attention(q, k, v, log_a, s0, lengths=ends)
    assert torch.equal(o, again_o) and torch.equal(s, again_s)


@pytest.mark.parametrize("decay", ["token", "strong"])
@pytest.mark.parametrize("shape,dtype,lengths", CASES, ids=str)
def test_gradients_over_cuts(ha, shape, dtype, lengths, decay):  # noqa: F811
    *ins, ends = inputs(shape, dtype, lengths, decay, 23 + sum(shape))
    wide = [leaf64(x) for x in (*clean(*ins[:4]), ins[4])]
    ins = [x.requires_grad_() for x in ins]
    o, s = ha.decay_attention(*ins, scale=0.25, lengths=ends)
    g = torch.Generator(device=DEV).manual_seed(3)
    d_o = torch.randn(o.shape, device=DEV, generator=g).to(dtype)
    d_s = torch.randn(s.shape, device=DEV, generator=g)
    want_o, want_s = attention64(*wide, scale=0.25, lengths=ends)
    got = torch.autograd.grad([o, s], ins, [d_o, d_s])
    want = torch.autograd.grad([want_o, want_s], wide, [d_o.double(), d_s.double()])
    for name, a, b in zip(("dq", "dk", "dv", "dlog_a", "dstate0"), got, want):
        close(a, b, name)


def test_state_in_place_over_cuts(ha):  # noqa: F811
    """The binding gives every call a state of its own; the C call may be given the first one."""
    q, k, v, log_a, s0 = make(1, 1400, 2, 2, 2, 2, 64, 64, BF16, state=True)
    o, s = ha.decay_attention(q, k, v, log_a, s0)
    own = s0.clone()
    p = ha._problem(q, k, v, log_a, own, 64 ** -0.5, None)
    out = torch.empty_like(o)
    ws = ha.workspace(q, k, v, log_a)
    ha._launch(q.device, ha._call().forward, p.packed, ha._ROWS.pack(*ha._rows(out, "o")), own.data_ptr(), ws.data_ptr(), ws.numel())
    assert torch.equal(out, o) and torch.equal(own, s)


@pytest.mark.parametrize("heads,kd,vd", [(1, 128, 128), (2, 40, 100), (5, 64, 32), (60, 64, 64), (80, 64, 128), (20, 64, 64)])
def test_steps_of_few_and_many_states(ha, heads, kd, vd):  # noqa: F811
    g = torch.Generator(device=DEV).manual_seed(5)
    q, k, v = (torch.randn(2, heads, d, device=DEV, generator=g) for d in (kd, kd, vd))
    log_a = -torch.rand(2, heads, device=DEV, generator=g)
    state = torch.randn(2, heads, kd, vd, device=DEV, generator=g)
    want = state.double() * log_a.double().exp()[..., None, None] + k.double().unsqueeze(-1) * v.double().unsqueeze(-2)
    o = ha.decay_attention_step(q, k, v, log_a, state)
    close(state, want, "state")
    close(o, kd ** -0.5 * (q.double().unsqueeze(-2) @ want).squeeze(-2), "o")


@pytest.mark.parametrize("dtype,t", [(BF16, 1400), (BF16, 100), (F32, 100)])
def test_a_kept_workspace_reports_no_fault(ha, dtype, t):  # noqa: F811
    from paper_2311_06281_b200 import heinsen_scan
    q, k, v, log_a, s0 = make(1, t, 2, 2, 2, 2, 64, 64, dtype, state=True)
    ws = ha.workspace(q, k, v, log_a)
    want = ha.decay_attention(q, k, v, log_a, s0)
    for fill in (0, 0xFF):  # its contents do not matter
        ws.fill_(fill)
        for _ in range(2):
            got = ha.decay_attention(q, k, v, log_a, s0, workspace=ws)
            heinsen_scan.check(ws)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(Exception, match="(?i)workspace"):
        ha.decay_attention(q, k, v, log_a, s0, workspace=ws[:256] if ws.numel() > 256 else ws[:0])
