"""The attention with a decay for each head against its float64 form, token by token: outputs, states and every gradient,
over types, head layouts, lengths from zero tokens to many chunks, strides, resets, ragged batches; the one-token step."""
import pytest
import torch

from attention_testlib import attention64, close, leaf64

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = "cuda"


@pytest.fixture(scope="module")
def ha():
    from paper_2311_06281_b200 import build_ext, heinsen_attention
    build_ext.build()
    heinsen_attention.lib()
    return heinsen_attention


def make(b, t, h, hq, hk, hv, kd, vd, dtype, decay="token", state=False, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s, to=dtype: torch.randn(*s, device=DEV, generator=g).to(to)  # noqa: E731
    q, k, v = rnd(b, t, hq, kd), rnd(b, t, hk, kd), rnd(b, t, hv, vd)
    if decay == "head":
        log_a = torch.log1p(-torch.exp2(-1 - 6 * torch.rand(h, device=DEV, generator=g)))
    elif decay == "strong":  # some steps forget nearly everything, some nothing
        log_a = -torch.exp(4 * torch.randn(b, t, h, device=DEV, generator=g))
    else:
        log_a = torch.nn.functional.logsigmoid(3 + torch.randn(b, t, h, device=DEV, generator=g))
        if decay == "reset":
            log_a = log_a.masked_fill(torch.rand(b, t, h, device=DEV, generator=g) < 0.04, -float("inf"))
    return q, k, v, log_a, rnd(b, h, kd, vd, to=F32) if state else None


SHAPES = [
    # b, t, h, hq, hk, hv, kd, vd
    (1, 1, 1, 1, 1, 1, 64, 64), (2, 2, 3, 3, 3, 3, 128, 128), (3, 17, 4, 4, 4, 4, 64, 64), (1, 32, 2, 2, 2, 2, 128, 64),
    (2, 127, 2, 2, 2, 2, 128, 128), (2, 128, 2, 2, 2, 2, 64, 128), (1, 129, 4, 2, 2, 4, 128, 128), (1, 300, 8, 8, 2, 2, 96, 64),
    (2, 257, 4, 1, 1, 4, 128, 80), (1, 515, 2, 2, 2, 2, 128, 128), (1, 40, 2, 1, 2, 1, 5, 3), (1, 70, 2, 2, 2, 2, 256, 256),
    (1, 130, 1, 1, 1, 1, 72, 136), (0, 5, 2, 2, 2, 2, 64, 64), (2, 0, 2, 2, 2, 2, 64, 64),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("decay,state", [("token", False), ("head", True), ("strong", True), ("reset", True)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(ha, shape, decay, state, dtype):
    q, k, v, log_a, s0 = make(*shape, dtype, decay, state, seed=sum(shape))
    o, s = ha.decay_attention(q, k, v, log_a, s0)
    want_o, want_s = attention64(q, k, v, log_a, s0, shape[6] ** -0.5)
    assert o.dtype == dtype and s.dtype == F32
    close(o, want_o, "o")
    close(s, want_s, "state")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("decay,state", [("token", False), ("head", True), ("strong", True)])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[1] <= 300], ids=str)
def test_gradients(ha, shape, decay, state, dtype):
    q, k, v, log_a, s0 = make(*shape, dtype, decay, state, seed=7 + sum(shape))
    ins = [x.requires_grad_() if x is not None else None for x in (q, k, v, log_a, s0)]
    o, s = ha.decay_attention(*ins, scale=0.25)
    g = torch.Generator(device=DEV).manual_seed(3)
    d_o = torch.randn(o.shape, device=DEV, generator=g).to(dtype)
    d_s = torch.randn(s.shape, device=DEV, generator=g) if state else None
    wide = [leaf64(x) for x in ins]
    want_o, want_s = attention64(*wide, scale=0.25)
    have = [i for i, x in enumerate(ins) if x is not None]
    got = torch.autograd.grad([o, s] if state else [o], [ins[i] for i in have], [d_o, d_s] if state else [d_o])
    want = torch.autograd.grad([want_o, want_s] if state else [want_o], [wide[i] for i in have],
                               [d_o.double(), d_s.double()] if state else [d_o.double()], allow_unused=True)
    for i, a, b in zip(have, got, want):
        name = ("dq", "dk", "dv", "dlog_a", "dstate0")[i]
        assert a.dtype == ins[i].dtype
        close(a, torch.zeros_like(wide[i]) if b is None else b, name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kd,vd", [(64, 64), (128, 128)])
def test_ragged_batch_never_reads_what_lies_behind_the_lengths(ha, kd, vd, dtype):
    b, t, h = 6, 261, 2
    q, k, v, log_a, s0 = make(b, t, h, h, h, h, kd, vd, dtype, state=True, seed=5)
    lengths = torch.tensor([0, 1, 128, 129, 261, 1000], dtype=torch.int32, device=DEV)
    for x in (q, k, v, log_a):
        for i, n in enumerate(lengths.tolist()):
            x[i, n:] = float("nan")
    ins = [x.requires_grad_() for x in (q, k, v, log_a, s0)]
    o, s = ha.decay_attention(*ins, lengths=lengths)
    d_o = torch.randn(o.shape, device=DEV).to(dtype)
    for i, n in enumerate(lengths.tolist()):
        d_o[i, n:] = float("nan")
    d_s = torch.randn(s.shape, device=DEV)
    got = torch.autograd.grad([o, s], ins, [d_o, d_s])
    clean = [leaf64(torch.nan_to_num(x)) for x in ins]
    want_o, want_s = attention64(*clean, scale=kd ** -0.5, lengths=lengths)
    close(o, want_o, "o")
    close(s, want_s, "state")
    want = torch.autograd.grad([want_o, want_s], clean, [torch.nan_to_num(d_o).double(), d_s.double()])
    for name, x, y in zip(("dq", "dk", "dv", "dlog_a", "dstate0"), got, want):
        close(x, y, name)
        if name != "dstate0":
            for i, n in enumerate(lengths.tolist()):
                assert (x[i, n:] == 0).all(), f"{name}: not zero behind the end of row {i}"
    assert torch.equal(s[0], s0[0].detach())  # no token: the state as it was


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_offsets(ha, dtype):
    """Views into one projected tensor, heads before tokens, an unaligned base: the same results as contiguous copies."""
    b, t, h, d = 2, 150, 3, 64
    fused = torch.randn(b, t, 3, h, d, device=DEV).to(dtype)
    log_a = torch.nn.functional.logsigmoid(2 + torch.randn(b, h, t, device=DEV)).transpose(1, 2)
    q, k, v = fused.unbind(2)
    plain = ha.decay_attention(q.contiguous(), k.contiguous(), v.contiguous(), log_a.contiguous())
    for views in ((q, k, v), tuple(x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (q, k, v)),
                  tuple(torch.cat([x, x[..., :1]], -1)[..., :d] for x in (q, k, v))):
        for got, want in zip(ha.decay_attention(*views, log_a), plain):
            close(got, want.double(), "a view")
    base = torch.randn(b * t * h * d + 1, device=DEV).to(dtype)[1:].view(b, t, h, d)  # not 16-byte aligned
    want, _ = attention64(base, k, v, log_a, None, d ** -0.5)
    close(ha.decay_attention(base, k, v, log_a)[0], want, "an unaligned base")
    one = torch.randn(1, 1, h, d, device=DEV).to(dtype).expand(b, t, h, d)  # strides of zero
    want, _ = attention64(one, k, v, log_a, None, d ** -0.5)
    close(ha.decay_attention(one, k, v, log_a)[0], want, "a broadcast query")


def test_gradients_of_views_and_expanded_decays(ha):
    torch.manual_seed(0)
    b, t, h, d = 2, 100, 2, 64
    fused = torch.randn(b, t, 3, h, d, device=DEV).to(BF16).requires_grad_()
    log_a = (-torch.rand(h, device=DEV)).requires_grad_()
    o, _ = ha.decay_attention(*fused.unbind(2), log_a.expand(b, t, h))
    d_o = torch.randn(o.shape, device=DEV).to(BF16).transpose(1, 2).contiguous().transpose(1, 2)
    got = torch.autograd.grad(o, (fused, log_a), d_o)
    f64, a64 = leaf64(fused), leaf64(log_a)
    want_o, _ = attention64(*f64.unbind(2), a64, None, d ** -0.5)
    for x, y in zip(got, torch.autograd.grad(want_o, (f64, a64), d_o.double())):
        close(x, y, "gradient")


def test_directional_differences(ha):
    """The gradients against central differences of the kernel's own forward pass, in float32."""
    q, k, v, log_a, s0 = make(2, 75, 4, 2, 4, 1, 24, 40, F32, state=True, seed=11)
    d_o, d_s = torch.randn(2, 75, 4, 40, device=DEV), torch.randn(2, 4, 24, 40, device=DEV)
    loss = lambda *x: sum((a.double() * w).sum() for a, w in zip(ha.decay_attention(*x), (d_o, d_s)))  # noqa: E731
    ins = [x.requires_grad_() for x in (q, k, v, log_a, s0)]
    grads = torch.autograd.grad(loss(*ins), ins)
    ins = [x.detach() for x in ins]
    for i, g in enumerate(grads):
        way = torch.randn_like(ins[i])
        step = 1e-2
        at = lambda e: loss(*[x + e * way if j == i else x for j, x in enumerate(ins)])  # noqa: E731
        with torch.no_grad():
            slope = float((at(step) - at(-step)) / (2 * step))
        want = float((g.double() * way).sum())
        # third-order term of the difference: linear in q, k, v, state0; the decays' is bounded by step^2 of the slope's scale
        size = float((g.double().abs() * way.abs()).sum()) / g.numel() ** 0.5
        assert abs(slope - want) <= 2e-2 * size, (i, slope, want, size)


def test_prompt_then_steps_equal_one_prompt(ha):
    """A prompt cut in two calls, and a prompt followed by single tokens, are the whole prompt."""
    q, k, v, log_a, s0 = make(2, 200, 4, 4, 2, 2, 64, 64, F32, state=True)
    whole, last = ha.decay_attention(q, k, v, log_a, s0)
    cut = lambda x, a, b: x[:, a:b]  # noqa: E731
    o1, s = ha.decay_attention(*(cut(x, 0, 133) for x in (q, k, v, log_a)), s0)
    close(o1, whole[:, :133].double(), "first part")
    pool = torch.full((5, 4, 64, 64), float("nan"), device=DEV)
    slots = torch.tensor([3, 1], dtype=torch.int32, device=DEV)
    pool[slots.long()] = s
    for t in range(133, 200):
        o = ha.decay_attention_step(q[:, t], k[:, t], v[:, t], log_a[:, t], pool, slots=slots)
        close(o, whole[:, t].double(), f"token {t}")
    close(pool[slots.long()], last.double(), "state")
    assert torch.isnan(pool[[0, 2, 4]]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("h,hq,hk,hv,kd,vd", [(4, 4, 4, 4, 128, 128), (8, 2, 2, 8, 64, 80), (6, 6, 3, 2, 96, 33), (1, 1, 1, 1, 1, 1),
                                              (2, 2, 2, 2, 256, 256), (3, 1, 3, 3, 7, 130)])
def test_step(ha, h, hq, hk, hv, kd, vd, dtype):
    b, pool = 5, 7
    q, k, v, log_a, _ = make(b, 1, h, hq, hk, hv, kd, vd, dtype, seed=kd)
    log_a[1, 0, 0] = -float("inf")
    state = torch.randn(pool, h, kd, vd, device=DEV)
    state[6, 0] = float("inf")  # forgotten by the decay of zero below
    slots = torch.tensor([2, 6, -1, 0, 7], dtype=torch.int32, device=DEV)
    if h > 1:
        state[6, 1:] = 1.0
    before = state.clone()
    o = ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], state, slots=slots, scale=0.3)
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < pool:
            want_o, want_s = attention64(q[i:i + 1], k[i:i + 1], v[i:i + 1], log_a[i:i + 1], before[s:s + 1], 0.3)
            close(o[i], want_o[0, 0], f"o of {i}")
            close(state[s], want_s[0], f"state of {i}")
        else:
            assert (o[i] == 0).all()
    untouched = [s for s in range(pool) if s not in slots.tolist()]
    assert torch.equal(state[untouched], before[untouched])


def test_step_with_fixed_decays_views_and_given_output(ha):
    b, h, d = 3, 2, 64
    fused = torch.randn(b, 3, h, d, device=DEV).to(BF16)
    q, k, v = fused.unbind(1)
    log_a = -torch.rand(h, device=DEV)
    state = torch.randn(b, h, d, d, device=DEV)
    want_o, want_s = attention64(q[:, None], k[:, None], v[:, None], log_a, state, d ** -0.5)
    out = torch.empty(b, h, d, dtype=BF16, device=DEV)
    assert ha.decay_attention_step(q, k, v, log_a, state, out=out) is out
    close(out, want_o[:, 0], "o")
    close(state, want_s, "state")


def test_other_streams_and_repeated_calls(ha):
    """Calls on a side stream see what that stream wrote before them; the same call gives the same bits."""
    q, k, v, log_a, s0 = make(2, 700, 4, 4, 4, 4, 128, 128, BF16, state=True)
    first = ha.decay_attention(q, k, v, log_a, s0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q2 = torch.zeros_like(q)
        q2.copy_(q)
        again = ha.decay_attention(q2, k, v, log_a, s0)
    side.synchronize()
    for x, y in zip(first, again):
        assert torch.equal(x, y)


def test_long_sequence_in_segments(ha):
    """A few heads and many tokens: the state at the end against chunks of the same call."""
    q, k, v, log_a, s0 = make(1, 20011, 2, 2, 2, 2, 128, 128, BF16, decay="head", state=True)
    o, s = ha.decay_attention(q, k, v, log_a, s0)
    at, parts = s0, []
    for lo in range(0, 20011, 1999):
        p, at = ha.decay_attention(*(x[:, lo:lo + 1999] for x in (q, k, v)), log_a, at)
        parts.append(p)
    close(o, torch.cat(parts, 1).double(), "o", rel=6 * 2.0 ** -9)
    close(s, at.double(), "state", rel=3e-5)
    # the last tokens from the definition: what lies 4000 tokens back weighs less than 2^-50 with windows up to 2^7
    tail_o, tail_s = attention64(*(x[:, -4000:] for x in (q, k, v)), log_a, None, 128 ** -0.5)
    close(o[:, -500:], tail_o[:, -500:], "last tokens")
    close(s, tail_s, "last state")


def test_refusals(ha):
    q, k, v, log_a, s0 = make(2, 8, 4, 4, 2, 2, 64, 64, BF16, state=True)
    ok = ha.decay_attention(q, k, v, log_a, s0)
    assert ok[0].shape == (2, 8, 4, 64)
    for bad in (lambda: ha.decay_attention(q, k[:, :4], v, log_a), lambda: ha.decay_attention(q, k, v, log_a[:, :, :3]),
                lambda: ha.decay_attention(q, k, v, log_a[0]), lambda: ha.decay_attention(q, k, v, log_a, s0[:, :2]),
                lambda: ha.decay_attention(q.transpose(-1, -2).contiguous().transpose(-1, -2), k, v, log_a),
                lambda: ha.decay_attention(q.cpu(), k.cpu(), v.cpu(), log_a.cpu()),
                lambda: ha.decay_attention(q, k, v, log_a, lengths=torch.ones(2, device=DEV)),
                lambda: ha.decay_attention(q[0], k[0], v[0], log_a),
                lambda: ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], s0[:1]),
                lambda: ha.decay_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], s0, slots=torch.zeros(2, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ha.decay_attention(q, k.float(), v, log_a), lambda: ha.decay_attention(q, k, v, log_a.to(BF16)),
                lambda: ha.decay_attention(q.half(), k.half(), v.half(), log_a), lambda: ha.decay_attention(q, k, v, log_a, s0.to(BF16))):
        with pytest.raises(TypeError):
            bad()
    for scale in (0.0, float("nan"), float("inf")):
        with pytest.raises((ValueError, ha.HeinsenScanError)):
            ha.decay_attention(q, k, v, log_a, scale=scale)
    big = torch.zeros(1, 2, 1, 257, device=DEV)
    with pytest.raises((ValueError, ha.HeinsenScanError)):
        ha.decay_attention(big, big, big, torch.zeros(1, 2, 1, device=DEV))
