"""decay_attention and the norms over the ranges they accept: gradients past resets, decays above one, what a NaN may spoil,
tensors whose offsets pass 2^31 elements; tolerances as in attention_testlib where nothing else is said."""
import pytest
import torch

from attention_testlib import attention64, close, leaf64
from test_gpu_attention import BF16, DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [(1, 128, 2, 2, 2, 2, 64, 64), (2, 300, 4, 2, 4, 1, 128, 72), (2, 257, 60, 60, 60, 60, 96, 128), (1, 900, 2, 1, 2, 2, 128, 128)]


def gradients_close(ha, ins, seed):  # noqa: F811
    wide = [leaf64(x) for x in ins]
    ins = [x.requires_grad_() for x in ins]
    got, want = ha.decay_attention(*ins, scale=0.25), attention64(*wide, scale=0.25)
    for name, a, b in zip(("o", "state"), got, want):
        close(a, b, name)
    g = torch.Generator(device=DEV).manual_seed(seed)
    d_o, d_s = (torch.randn(x.shape, device=DEV, generator=g).to(x.dtype) for x in got)
    got = torch.autograd.grad(got, ins, [d_o, d_s])
    want = torch.autograd.grad(want, wide, [d_o.double(), d_s.double()])
    for name, a, b in zip(("dq", "dk", "dv", "dlog_a", "dstate0"), got, want):
        close(a, b, name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients_past_resets(ha, shape, dtype):  # noqa: F811
    gradients_close(ha, make(*shape, dtype, "reset", True, seed=sum(shape)), 5)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_decays_above_one(ha, shape, dtype):  # noqa: F811
    """Log decays of both signs; within 128 tokens their sums stay below 0.02 * 128 + 0.1 * 60 in size, over all tokens below 40."""
    q, k, v, log_a, s0 = make(*shape, dtype, state=True, seed=1 + sum(shape))
    g = torch.Generator(device=DEV).manual_seed(8)
    log_a = (0.02 + 0.1 * torch.randn(log_a.shape, device=DEV, generator=g)).masked_fill(
        torch.rand(log_a.shape, device=DEV, generator=g) < 0.005, -float("inf"))
    sums = log_a.masked_fill(log_a == -float("inf"), 0.0).cumsum(1)
    assert float(sums.max() - sums.min()) < 40
    gradients_close(ha, [q, k, v, log_a, s0], 6)


@pytest.mark.parametrize("dtype,chunk", [(BF16, 128), (F32, 32)])
@pytest.mark.parametrize("b,t,h", [(2, 300, 2), (2, 300, 40)])
def test_what_a_nan_spoils(ha, b, t, h, dtype, chunk):  # noqa: F811
    """Its own head of its own row, from the beginning of its chunk on; nothing else."""
    q, k, v, log_a, s0 = make(b, t, h, h, h, h, 64, 64, dtype, state=True, seed=9)
    want, last = ha.decay_attention(q, k, v, log_a, s0)
    for x in (q, k, v, log_a):
        spoilt = [y.clone() for y in (q, k, v, log_a)]
        which = [y is x for y in (q, k, v, log_a)].index(True)
        spoilt[which][1, 200, 1] = float("nan")
        o, s = ha.decay_attention(*spoilt, s0)
        same = torch.ones(b, t, h, dtype=torch.bool, device=DEV)
        same[1, 200 // chunk * chunk:, 1] = False
        assert torch.equal(o[same], want[same])
        others = torch.ones(b, h, dtype=torch.bool, device=DEV)
        others[1, 1] = False
        assert torch.equal(s[others], last[others])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dims", [(64, 64), (128, 72)])
@pytest.mark.parametrize("which", ["batch", "token"])
def test_offsets_past_31_bits(ha, which, dims, dtype):  # noqa: F811
    """Views whose rows lie 2^31 elements and more apart give the bits that contiguous copies give."""
    h, far = 2, (1 << 31) + 8 if which == "batch" else 1 << 30
    b, t = (2, 40) if which == "batch" else (1, 4)
    small = [*make(b, t, h, h, h, h, *dims, dtype, seed=3)[:3], torch.randn(b, t, h, dims[1], device=DEV).to(dtype)]
    base = torch.empty((b - 1) * far + (1 << 16) if which == "batch" else (t - 1) * far + (1 << 16), dtype=dtype, device=DEV)
    views, at = [], 0
    for x in small:
        d, room = x.shape[-1], x[0, 0].numel() if which == "token" else x[0].numel()
        strides = (far, h * d, d, 1) if which == "batch" else (0, far, d, 1)
        views.append(base.as_strided(x.shape, strides, at))
        views[-1].copy_(x)
        at += room
    assert at < 1 << 16
    log_a = -torch.rand(b, t, h, device=DEV)
    results = []
    for q, k, v, d_o in (small, views):
        ins = [x.detach().requires_grad_() for x in (q, k, v, log_a)]
        o, s = ha.decay_attention(*ins)
        results.append((o, s, *torch.autograd.grad(o, ins, d_o)))
    for a, b_ in zip(*results):
        assert torch.equal(a, b_)


def test_a_pool_of_states_past_31_bits(ha):  # noqa: F811
    n = (1 << 16) + 5  # rows of 2 * 128 * 128: more than 2^31 elements
    q, k, v, log_a, _ = make(3, 1, 2, 2, 2, 2, 128, 128, BF16, seed=4)
    pool = torch.empty(n, 2, 128, 128, device=DEV)
    slots = torch.tensor([n - 1, 0, n - 3], dtype=torch.int32, device=DEV)
    states = torch.randn(3, 2, 128, 128, device=DEV)
    pool[slots.long()] = states
    o = ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], pool, slots=slots)
    want = ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], states)
    assert torch.equal(o, want) and torch.equal(pool[slots.long()], states)


def test_norms_past_31_bits(ha):  # noqa: F811
    rows, d = (1 << 20) + 3, 2048
    x = torch.randn(1 << 16, d, device=DEV).to(BF16).repeat(17, 1)[:rows]
    w = torch.rand(d, device=DEV).to(BF16)
    last = x[-5:].clone().requires_grad_()
    x.requires_grad_()
    for call in (lambda t: ha.block_norms(t, t, w, post_weight=w)[1], lambda t: ha.gated_norm(t, t, w)):
        y, want = call(x), call(last)
        assert torch.equal(y[-5:], want)
        dy = torch.ones((), device=DEV, dtype=BF16).expand(rows, d)
        got, = torch.autograd.grad(y, x, dy)
        del y
        back, = torch.autograd.grad(want, last, dy[:5])
        assert torch.equal(got[-5:], back)
        del got
