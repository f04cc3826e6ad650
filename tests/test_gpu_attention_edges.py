"""decay_attention and the norms at the edges of what they accept: foreign workspaces, empty batches, states that a decay of
zero has to forget, derivatives and in-place updates as autograd sees them."""
import pytest
import torch

from attention_testlib import attention64, close, leaf64
from test_gpu_attention import BF16, DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu


def test_a_workspace_of_the_host_is_refused(ha):  # noqa: F811
    q, k, v, log_a, s0 = make(1, 40, 2, 2, 2, 2, 64, 64, BF16, state=True)
    ws = ha.workspace(q, k, v, log_a)
    for bad in (ws.cpu(), torch.empty(ws.numel(), device=DEV)):
        for grad in (False, True):
            with pytest.raises(ValueError, match="workspace"):
                ha.decay_attention(q.detach().requires_grad_(grad), k, v, log_a, s0, workspace=bad)


def leave_nan_behind(*shapes):
    """Fills what the allocator will hand out next: a result that nobody writes is NaN then, not a zero by chance."""
    kept = [torch.full(s, float("nan"), device=DEV) for s in shapes for _ in range(16)]
    torch.cuda.synchronize()
    del kept


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_of_an_empty_batch_are_zero(ha, dtype):  # noqa: F811
    q = torch.empty(0, 5, 2, 64, device=DEV, dtype=dtype, requires_grad=True)
    log_a = (-torch.rand(2, device=DEV)).requires_grad_()
    o, s = ha.decay_attention(q, q, q, log_a)
    leave_nan_behind((2,), (64,))
    dq, da = torch.autograd.grad(o.sum() + s.sum(), (q, log_a))
    assert dq.shape == q.shape and torch.equal(da, torch.zeros_like(log_a))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("fixed", [False, True])
def test_gradients_without_heads_are_zero(ha, fixed, dtype):  # noqa: F811
    q, k, v = (torch.randn(2, 3, 1, 16, device=DEV).to(dtype).requires_grad_() for _ in range(3))
    log_a = torch.empty((0,) if fixed else (2, 3, 0), device=DEV, requires_grad=True)
    o, s = ha.decay_attention(q, k, v, log_a)
    assert o.shape == (2, 3, 0, 16) and s.shape == (2, 0, 16, 16)
    leave_nan_behind(q.shape, (q.numel() // 2,))
    for g, x in zip(torch.autograd.grad(o.sum() + s.sum(), (q, k, v, log_a)), (q, k, v, log_a)):
        assert torch.equal(g, torch.zeros_like(x))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_of_sequences_without_tokens_have_zero_gradients(ha, dtype):  # noqa: F811
    x, branch = (torch.empty(3, 0, 64, device=DEV, dtype=dtype, requires_grad=True) for _ in range(2))
    gate = torch.randn(3, 1, 64, device=DEV).to(dtype).requires_grad_()
    pre, post = (torch.ones(64, device=DEV, dtype=dtype, requires_grad=True) for _ in range(2))
    r, y = ha.block_norms(x, branch, pre, post_weight=post, gate=gate)
    leave_nan_behind((64,), (32,), (192,), (96,))
    ins = (x, branch, gate, pre, post)
    for g, t in zip(torch.autograd.grad(r.sum() + y.sum(), ins), ins):
        assert torch.equal(g, torch.zeros_like(t))


# (b, t, h, kd, vd): whole, and cut into segments (bf16 at multiples of 128 tokens, float32 of 32)
FORGET = [(2, 300, 60, 64, 64), (2, 300, 2, 128, 72), (1, 1500, 2, 64, 128)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("at", [0, 50, 127, 128, 200])
@pytest.mark.parametrize("b,t,h,kd,vd", FORGET)
def test_a_decay_of_zero_forgets_whatever_the_state_holds(ha, b, t, h, kd, vd, at, dtype):  # noqa: F811
    q, k, v, log_a, s0 = make(b, t, h, h, h, h, kd, vd, dtype, state=True, seed=at)
    log_a[:, at] = -float("inf")
    s0[:, :, 0] = float("nan")
    s0[:, :, 1, 1:] = float("inf")
    s0[:, :, 2, ::2] = -float("inf")
    o, s = ha.decay_attention(q, k, v, log_a, s0)
    want_o, want_s = attention64(*(x[:, at:] for x in (q, k, v, log_a)), None, kd ** -0.5)
    close(o[:, at:], want_o, "o")
    close(s, want_s, "state")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,t,h,kd,vd", FORGET[1:])
def test_gradients_past_a_forgotten_state(ha, b, t, h, kd, vd, dtype):  # noqa: F811
    q, k, v, log_a, s0 = make(b, t, h, h, h, h, kd, vd, dtype, state=True, seed=1)
    log_a[:, 0] = -float("inf")
    g = torch.Generator(device=DEV).manual_seed(3)
    d_o, d_s = torch.randn(b, t, h, vd, device=DEV, generator=g).to(dtype), torch.randn(b, h, kd, vd, device=DEV, generator=g)
    wide = [leaf64(x) for x in (q, k, v, log_a, s0)]
    want = torch.autograd.grad(attention64(*wide, scale=0.25), wide, [d_o.double(), d_s.double()])
    s0[:, :, 0], s0[:, :, 1, 1:] = float("nan"), float("inf")
    ins = [x.requires_grad_() for x in (q, k, v, log_a, s0)]
    got = torch.autograd.grad(ha.decay_attention(*ins, scale=0.25), ins, [d_o, d_s])
    for name, x, y in zip(("dq", "dk", "dv", "dlog_a", "dstate0"), got, want):
        close(x, y, name)
    assert (got[4] == 0).all()


def pairs_weight(q, k, v, log_a, d_o, scale, chunk):
    """The sum of |W_ij| over the pairs i >= j of every chunk, for every token of it: what a sum over them can be off by."""
    q, k, v, a, g = (x.double().transpose(1, 2) for x in (q, k, v, log_a.unsqueeze(-1), d_o))
    out = torch.zeros(*log_a.shape, dtype=torch.float64, device=log_a.device)
    for t0 in range(0, q.shape[2], chunk):
        at = slice(t0, t0 + chunk)
        c = a[:, :, at, 0].clamp(min=-1e4).cumsum(-1)
        w = torch.exp((c[..., :, None] - c[..., None, :]).tril()).tril() * scale
        w = (w * (q[:, :, at] @ k[:, :, at].mT) * (g[:, :, at] @ v[:, :, at].mT)).abs().sum((-1, -2))
        out[:, at] = w[:, None]
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,t,h,kd,vd", [(1, 128, 2, 64, 64), (2, 300, 60, 128, 128), (2, 300, 2, 128, 72), (1, 1500, 2, 64, 128)])
def test_decay_gradients_where_decays_are_strong(ha, b, t, h, kd, vd, dtype):  # noqa: F811
    """A few tokens forget all or nearly all (-inf, -20): their own gradients, not only those beside them.  Nothing crosses a
    reset, so its gradient is zero but for the sums of what lies on both sides of it: with sums over up to 2 * 128 products
    on each of two sides in 64 bits that is 512 * 2^-53 of the products' absolute sum.  The others are held to float32's
    tolerance by themselves."""
    q, k, v, log_a, s0 = make(b, t, h, h, h, h, kd, vd, dtype, state=True, seed=2)
    g = torch.Generator(device=DEV).manual_seed(4)
    which = torch.rand(b, t, h, device=DEV, generator=g)
    reset, strong = which < 0.02, (which >= 0.02) & (which < 0.04)
    log_a = log_a.masked_fill(reset, -float("inf")).masked_fill(strong, -20.0)
    d_o, d_s = torch.randn(b, t, h, vd, device=DEV, generator=g).to(dtype), torch.randn(b, h, kd, vd, device=DEV, generator=g)
    ins, wide = [x.requires_grad_() for x in (q, k, v, log_a, s0)], [leaf64(x) for x in (q, k, v, log_a, s0)]
    got, = torch.autograd.grad(ha.decay_attention(*ins, scale=0.25), log_a, [d_o, d_s])
    want, = torch.autograd.grad(attention64(*wide, scale=0.25), wide[3], [d_o.double(), d_s.double()])
    close(got, want, "dlog_a")
    bound = pairs_weight(q.detach(), k.detach(), v.detach(), log_a.detach(), d_o, 0.25, 128) * 2.0 ** -44
    assert reset.any() and strong.any() and (want[reset] == 0).all()
    worst = float((got[reset].double().abs() / bound[reset]).max())
    assert worst <= 1, f"at a reset: {float(got[reset].abs().max()):.3g}, {worst:.3g} times what sums in 64 bits may leave"
    close(got[strong], want[strong], "dlog_a at strong decays")


def test_a_step_on_a_state_that_a_graph_has_kept_is_noticed(ha):  # noqa: F811
    q, k, v, log_a, s0 = make(2, 9, 2, 2, 2, 2, 64, 64, F32, state=True)
    q.requires_grad_()
    one = [x[:, 0].detach() for x in (q, k, v, log_a)]
    o, _ = ha.decay_attention(q, k, v, log_a, s0)
    before, out = s0._version, torch.empty(2, 2, 64, device=DEV)
    ha.decay_attention_step(*one, s0, out=out)
    assert s0._version > before and out._version > 0
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(o.sum(), q)
    kept = (out.clone().requires_grad_() * out).sum()  # its backward needs `out`
    ha.decay_attention_step(*one, s0, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
    with torch.inference_mode():  # tensors without a version
        state = s0.clone()
        ha.decay_attention_step(*one, state)


def test_tangents_are_refused_and_not_dropped(ha):  # noqa: F811
    from torch.autograd import forward_ad
    q, k, v, log_a, s0 = make(2, 9, 2, 2, 2, 2, 64, 64, F32, state=True)
    x, w = torch.randn(4, 64, device=DEV), torch.ones(64, device=DEV)
    want = [*ha.decay_attention(q, k, v, log_a, s0), *ha.block_norms(x, x, w), ha.gated_norm(x, x, w)]
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))  # noqa: E731
        for call in (lambda: ha.decay_attention(dual(q), k, v, log_a), lambda: ha.decay_attention(q, k, v, log_a, dual(s0)),
                     lambda: ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], dual(log_a[:, 0]), s0.clone()),
                     lambda: ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], dual(s0.clone())),
                     lambda: ha.block_norms(x, dual(x), w), lambda: ha.block_norms(x, x, w, gate=dual(x)),
                     lambda: ha.gated_norm(x, x, dual(w))):
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(NotImplementedError):
                    call()
        # without a tangent nothing changes while a level is active
        got = [*ha.decay_attention(q, k, v, log_a, s0), *ha.block_norms(x, x, w), ha.gated_norm(x, x, w)]
        ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], s0.clone())
    for a, b in zip(got, want):
        assert torch.equal(a, b)
