"""The delta rule with a decay against its float64 form, token by token: outputs, states and every gradient, over types, head
layouts, lengths from zero tokens to many chunks, strides, resets, ragged batches, few and many sequences (the two kinds of pass);
the one-token step."""
import pytest
import torch

from attention_testlib import close, leaf64
from delta_testlib import delta64

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DEV = "cuda"


@pytest.fixture(scope="module")
def hd():
    from paper_2311_06281_b200 import build_ext, heinsen_delta
    build_ext.build()
    heinsen_delta.lib()
    return heinsen_delta


def make(b, t, h, hq, hk, hv, kd, vd, dtype, decay="token", state=False, seed=0, most=1.0):
    """Keys of length one and beta below `most`, as layers of this kind have them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s, to=dtype: torch.randn(*s, device=DEV, generator=g).to(to)  # noqa: E731
    q, v = rnd(b, t, hq, kd), rnd(b, t, hv, vd)
    k = torch.nn.functional.normalize(rnd(b, t, hk, kd, to=F32), dim=-1).to(dtype)
    beta = most * torch.sigmoid(2 * rnd(b, t, h, to=F32))
    if decay == "head":
        log_a = torch.log1p(-torch.exp2(-1 - 6 * torch.rand(h, device=DEV, generator=g)))
    elif decay == "strong":  # some steps forget nearly everything, some nothing
        log_a = -torch.exp(4 * torch.randn(b, t, h, device=DEV, generator=g))
    elif decay == "none":
        log_a = torch.zeros(h, device=DEV)
    else:
        log_a = torch.nn.functional.logsigmoid(3 + torch.randn(b, t, h, device=DEV, generator=g))
        if decay == "reset":
            log_a = log_a.masked_fill(torch.rand(b, t, h, device=DEV, generator=g) < 0.04, -float("inf"))
    return q, k, v, log_a, beta, rnd(b, h, kd, vd, to=F32) if state else None


NAMES = ("dq", "dk", "dv", "dlog_a", "dbeta", "dstate0")
SHAPES = [
    # b, t, h, hq, hk, hv, kd, vd
    (1, 1, 1, 1, 1, 1, 64, 64), (2, 2, 3, 3, 3, 3, 128, 128), (3, 17, 4, 4, 4, 4, 64, 64), (2, 63, 2, 2, 2, 2, 128, 128),
    (2, 64, 2, 2, 2, 2, 64, 128), (1, 65, 4, 2, 2, 4, 128, 128), (1, 300, 8, 8, 2, 2, 96, 64), (2, 257, 4, 1, 1, 4, 128, 80),
    (1, 40, 2, 1, 2, 1, 5, 3), (1, 70, 2, 2, 2, 2, 256, 256), (1, 130, 1, 1, 1, 1, 72, 136), (2, 33, 2, 2, 2, 1, 129, 17),
    (0, 5, 2, 2, 2, 2, 64, 64), (2, 0, 2, 2, 2, 2, 64, 64),
    # many slices of values: the other kind of pass
    (3, 130, 16, 16, 16, 16, 64, 128), (3, 65, 16, 8, 8, 16, 128, 136),
]
# ... of which for the gradients
MANY = [(5, 70, 16, 16, 16, 16, 64, 128), (5, 67, 16, 8, 4, 16, 128, 104), (5, 65, 16, 16, 16, 8, 96, 144)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("decay,state", [("token", False), ("head", True), ("strong", True), ("reset", True)])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(hd, shape, decay, state, dtype):
    q, k, v, log_a, beta, s0 = make(*shape, dtype, decay, state, seed=sum(shape))
    o, s = hd.delta_attention(q, k, v, log_a, beta, s0)
    want_o, want_s = delta64(q, k, v, log_a, beta, s0, shape[6] ** -0.5)
    assert o.dtype == dtype and s.dtype == F32
    close(o, want_o, "o")
    close(s, want_s, "state")
    hd.check(DEV)


def gradients(hd, ins, scale, state, dtype, lengths=None):
    o, s = hd.delta_attention(*ins, scale=scale, lengths=lengths)
    g = torch.Generator(device=DEV).manual_seed(3)
    d_o = torch.randn(o.shape, device=DEV, generator=g).to(dtype)
    d_s = torch.randn(s.shape, device=DEV, generator=g) if state else None
    wide = [leaf64(x) for x in ins]
    want_o, want_s = delta64(*wide, scale=scale, lengths=lengths)
    have = [i for i, x in enumerate(ins) if x is not None]
    got = torch.autograd.grad([o, s] if state else [o], [ins[i] for i in have], [d_o, d_s] if state else [d_o])
    want = torch.autograd.grad([want_o, want_s] if state else [want_o], [wide[i] for i in have],
                               [d_o.double(), d_s.double()] if state else [d_o.double()], allow_unused=True)
    for i, a, b in zip(have, got, want):
        assert a.dtype == ins[i].dtype
        b = torch.zeros_like(wide[i]) if b is None else b
        # a log decay of -inf has no effect through which a gradient could come (0 * inf in the plain form)
        close(a, torch.nan_to_num(b) if i == 3 else b, NAMES[i])
    hd.check(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("decay,state", [("token", False), ("head", True), ("strong", True)])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] * s[2] < 40], ids=str)
def test_gradients(hd, shape, decay, state, dtype):
    ins = [x.requires_grad_() if x is not None else None for x in make(*shape, dtype, decay, state, seed=7 + sum(shape))]
    gradients(hd, ins, 0.25, state, dtype)


@pytest.mark.parametrize("decay,state", [("token", True), ("head", False), ("strong", True)])
@pytest.mark.parametrize("shape", MANY, ids=str)
def test_gradients_of_many_sequences(hd, shape, decay, state):
    ins = [x.requires_grad_() if x is not None else None for x in make(*shape, BF16, decay, state, seed=7 + sum(shape))]
    gradients(hd, ins, 0.25, state, BF16)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(4, 200, 2, 2, 2, 2, 64, 64), (5, 150, 16, 8, 8, 16, 64, 128)], ids=str)
def test_sequences_of_different_lengths(hd, shape, dtype):
    """What lies behind a sequence's end is never used, whatever it holds; outputs and gradients are zero there."""
    ins = make(*shape, dtype, "token", True, seed=5)
    ends = torch.tensor([0, 1, 64, 130, shape[1]][:shape[0]], dtype=torch.int32, device=DEV)
    behind = torch.arange(shape[1], device=DEV) >= ends[:, None]
    for x in ins[:5]:
        x.masked_fill_(behind.view(*behind.shape, *[1] * (x.dim() - 2)), float("nan"))
    clean = [torch.nan_to_num(x).requires_grad_() for x in ins]
    ins = [x.requires_grad_() for x in ins]
    got, want = hd.delta_attention(*ins, lengths=ends), delta64(*clean, scale=shape[6] ** -0.5, lengths=ends)
    for a, b, n in zip(got, want, ("o", "state")):
        close(a, b, n)
    d_o = torch.randn(got[0].shape, device=DEV).to(dtype)
    d_o[behind] = float("nan")
    d_s = torch.randn(got[1].shape, device=DEV)
    grads = torch.autograd.grad(got, ins, [d_o, d_s])
    wide = [leaf64(x) for x in clean]
    want = torch.autograd.grad(delta64(*wide, scale=shape[6] ** -0.5, lengths=ends), wide, [torch.nan_to_num(d_o).double(), d_s.double()])
    for a, b, n in zip(grads, want, NAMES):
        close(a, b, n)
    assert all((x[behind] == 0).all() for x in (got[0], *grads[:5]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("most,same", [(0.0, False), (1.0, True), (2.0, False)])
def test_extreme_writes(hd, dtype, most, same):
    """Nothing is written (beta 0), every token writes to the same key, errors are written twice over."""
    q, k, v, log_a, beta, s0 = make(1, 150, 2, 2, 2, 2, 64, 64, dtype, "none", True, seed=2, most=most)
    if same:
        k = k[:, :1].expand_as(k).contiguous()
        beta = torch.ones_like(beta)
    gradients(hd, [x.requires_grad_() for x in (q, k, v, log_a, beta, s0)], 0.25, True, dtype)


@pytest.mark.parametrize("shape", [(2, 200, 2, 2, 2, 2, 64, 64), (5, 150, 16, 16, 16, 16, 64, 128)], ids=str)
def test_decay_gradients_where_decays_are_strong(hd, shape):
    """All decays 2^-20: nothing but what passes over a token may be left in its decay's gradient."""
    ins = [x.requires_grad_() for x in make(*shape, BF16, "token", True, seed=4)]
    ins[3] = torch.full_like(ins[3], -14.0).requires_grad_()
    gradients(hd, ins, 0.25, True, BF16)


@pytest.mark.parametrize("shape", [(2, 100, 2, 2, 2, 2, 64, 64), (5, 100, 16, 16, 16, 16, 64, 128)], ids=str)
def test_a_decay_of_zero_forgets_whatever_the_state_holds(hd, shape):
    q, k, v, log_a, beta, s0 = make(*shape, BF16, "token", True, seed=8)
    log_a[:, 0] = -float("inf")
    want = hd.delta_attention(q, k, v, log_a, beta, torch.zeros_like(s0))
    s0[:] = float("nan")
    got = hd.delta_attention(q, k, v, log_a, beta, s0)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strides_and_alignments(hd, dtype):
    """Tensors cut out of others, at odd places, with expanded heads and gates: the same as their copies."""
    g = torch.Generator(device=DEV).manual_seed(1)
    b, t, h, d = 2, 90, 4, 64
    big = torch.randn(b, t + 3, 3 * h, d + 3, device=DEV, generator=g).to(dtype)
    q, k, v = big[:, 1:-2, :h, 1:-2], big[:, 2:-1, h:2 * h, 2:-1], big[:, 3:, 2 * h:, 3:]
    k = torch.nn.functional.normalize(k.float(), dim=-1).to(dtype)
    wide = torch.zeros(b, h, t, 2 * d + 2, device=DEV, dtype=dtype)
    wide[..., 1:d + 1] = k.transpose(1, 2)
    k = wide[..., 1:d + 1].transpose(1, 2)
    log_a = -torch.rand(b, 1, h, device=DEV, generator=g).expand(b, t, h)
    beta = torch.rand(t, h, device=DEV, generator=g).expand(b, t, h)
    v = v[:, :, :1].expand(b, t, h, d)
    ins = [x.requires_grad_() for x in (q.detach(), k.detach(), v.detach(), log_a.detach(), beta.detach())]
    copies = [x.detach().clone().contiguous().requires_grad_() for x in ins]
    d_o = torch.randn(b, h, t, d, device=DEV, generator=g).to(dtype).transpose(1, 2)
    outs = []
    for x in (ins, copies):
        o, s = hd.delta_attention(*x)
        outs.append([o, s, *torch.autograd.grad(o, x, d_o)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_against_differences(hd, dtype):
    """Along the gradient itself the loss changes by the step times its length; float32 throughout, h ~ eps^(1/3): 1e-2."""
    ins = [x.requires_grad_() for x in make(1, 75, 2, 1, 2, 2, 64, 64, F32, "token", True, seed=9)]
    if dtype == BF16:  # the point at which the bfloat16 kernels are asked, on its grid
        ins = [x.detach().to(BF16).float().requires_grad_() if i < 3 else x for i, x in enumerate(ins)]
    def loss(xs):
        o, s = hd.delta_attention(*xs)
        return (o.double() * torch.sin(torch.arange(o.numel(), device=DEV).view_as(o).double())).sum() + s.double().pow(2).sum()
    at = [x.detach().to(dtype).requires_grad_() if i < 3 else x.detach().requires_grad_() for i, x in enumerate(ins)]
    grads = [g.double() for g in torch.autograd.grad(loss(at), at)]
    size = torch.stack([g.pow(2).sum() for g in grads]).sum().sqrt()
    h = 3e-3
    ends = [loss([(x.detach().double() + sign * h * g / size).float() for x, g in zip(ins, grads)]) for sign in (1, -1)]
    assert abs(float((ends[0] - ends[1]) / (2 * h) / size) - 1) < 1e-2


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("b,h,hq,hk,hv,kd,vd", [(1, 1, 1, 1, 1, 1, 1), (3, 4, 2, 1, 4, 64, 64), (40, 16, 16, 16, 16, 128, 128),
                                               (2, 3, 3, 3, 3, 256, 256), (5, 2, 2, 2, 2, 33, 31), (70, 4, 4, 4, 4, 200, 68)])
def test_step(hd, b, h, hq, hk, hv, kd, vd, dtype):
    q, k, v, log_a, beta, pool = make(b + 3, 1, h, hq, hk, hv, kd, vd, dtype, "token", True, seed=b)
    q, k, v, log_a, beta = (x[:b, 0] for x in (q, k, v, log_a, beta))
    slots = torch.randperm(b + 3, device=DEV)[:b].to(torch.int32)
    before = pool.clone()
    o = hd.delta_attention_step(q, k, v, log_a, beta, pool, slots=slots)
    want_o, want_s = delta64(*(x.unsqueeze(1) for x in (q, k, v, log_a, beta)), before[slots.long()], scale=kd ** -0.5)
    close(o, want_o[:, 0], "o")
    close(pool[slots.long()], want_s, "state")
    rest = torch.ones(b + 3, dtype=torch.bool, device=DEV)
    rest[slots.long()] = False
    assert torch.equal(pool[rest], before[rest])


def test_steps_without_a_slot(hd):
    q, k, v, log_a, beta, pool = make(4, 1, 2, 2, 2, 2, 64, 64, BF16, "token", True)
    before = pool.clone()
    out = torch.full((4, 2, 64), float("nan"), device=DEV, dtype=BF16)
    o = hd.delta_attention_step(q[:, 0], k[:, 0], v[:, 0], log_a[:, 0], beta[:, 0], pool, out=out,
                                slots=torch.tensor([-1, 2, 4, 1 << 30], dtype=torch.int32, device=DEV))
    assert o is out and (o[[0, 2, 3]] == 0).all() and torch.isfinite(o[1]).all()
    assert torch.equal(pool[[0, 1, 3]], before[[0, 1, 3]]) and not torch.equal(pool[2], before[2])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens", [1, 70])
def test_steps_continue_a_prompt(hd, tokens, dtype):
    q, k, v, log_a, beta, s0 = make(2, tokens + 6, 4, 2, 2, 4, 64, 80, dtype, "token", True, seed=6)
    want_o, want_s = delta64(q, k, v, log_a, beta, s0, 0.125)
    _, state = hd.delta_attention(*(x[:, :tokens] for x in (q, k, v, log_a, beta)), s0, scale=0.125)
    for i in range(tokens, tokens + 6):
        o = hd.delta_attention_step(*(x[:, i] for x in (q, k, v, log_a, beta)), state, scale=0.125)
        close(o, want_o[:, i], "o")
    close(state, want_s, "state")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_32_bits(hd, dtype):
    """Batches and tokens more than 2^31 elements apart, and states behind 2^31 elements of a pool."""
    far = torch.empty(((1 << 31) + (1 << 22)) * (2 if dtype is F32 else 1) + (1 << 22), device=DEV, dtype=BF16).view(dtype)
    q, k, v, log_a, beta, state = make(2, 70, 2, 2, 2, 2, 64, 64, dtype, "token", True, seed=3)
    wide = [far.as_strided(x.shape, ((1 << 31) + 8 * n, 192 * 2 * 64, 64, 1), 64 * 2 * 64 * n) for n, x in enumerate((q, k, v))]
    for to, x in zip(wide, (q, k, v)):
        to.copy_(x)
    ins = [x.detach().requires_grad_() for x in (*wide, log_a, beta, state)]
    plain = [x.detach().requires_grad_() for x in (q, k, v, log_a, beta, state)]
    outs = []
    for x in (ins, plain):
        o, s = hd.delta_attention(*x)
        outs.append([o, s, *torch.autograd.grad((o.float().sum() + s.sum()), x)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    pool = torch.empty((1 << 31) // (2 * 64 * 64) + 2, 2, 64, 64, device=DEV)
    slots = torch.tensor([pool.shape[0] - 1, 0], dtype=torch.int32, device=DEV)
    pool[slots.long()] = state
    step = [x[:, 0] for x in (q, k, v, log_a, beta)]
    got = hd.delta_attention_step(*(x[:, 0] for x in wide), *step[3:], pool, slots=slots)
    assert torch.equal(got, hd.delta_attention_step(*step, state)) and torch.equal(pool[slots.long()], state)


def test_a_kept_workspace_and_a_captured_call(hd):
    """Two graphs of the same call on one workspace, replayed in turn with new inputs, beside an eager call on another stream."""
    from paper_2311_06281_b200 import heinsen_scan as hs
    ins = list(make(2, 150, 4, 4, 4, 4, 64, 64, BF16, "token", True, seed=1))
    other = make(2, 150, 4, 4, 4, 4, 64, 64, BF16, "token", True, seed=2)
    ws = hd.workspace(*ins[:5])
    want = [hd.delta_attention(*x) for x in (ins, other)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(hd.delta_attention(*ins, workspace=ws))
        graphs.append(graph)
    side = torch.cuda.Stream()
    first = [x.clone() for x in ins]
    for values, expected in ((other, want[1]), (first, want[0])):
        for x, y in zip(ins, values):
            x.copy_(y)
        for graph in graphs:
            graph.replay()
        with torch.cuda.stream(side):
            eager = hd.delta_attention(*other)
        torch.cuda.synchronize()
        for got in outs:
            assert all(torch.equal(a, b) for a, b in zip(got, expected))
        assert all(torch.equal(a, b) for a, b in zip(eager, want[1]))
    hs.check(ws)


def test_a_training_step_is_captured(hd):
    ins = [x.requires_grad_() for x in make(2, 100, 4, 2, 2, 4, 64, 64, BF16, "head", True, seed=1)]
    d_o = torch.randn(2, 100, 4, 64, device=DEV).to(BF16)

    def step():
        o, _ = hd.delta_attention(*ins)
        return torch.autograd.grad(o, ins, d_o)
    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_what_autograd_sees(hd):
    ins = list(make(1, 9, 2, 2, 2, 2, 64, 64, F32, "head", True))
    only = ins[4].requires_grad_()  # beta alone
    o, s = hd.delta_attention(*ins)
    (g,) = torch.autograd.grad(s.sum(), [only])  # through the state alone
    wide = [leaf64(x) for x in ins]
    close(g, torch.autograd.grad(delta64(*wide, scale=64 ** -0.5)[1].sum(), wide[4])[0], "dbeta")
    state = ins[5].detach().clone()
    kept = (state * state.clone().requires_grad_()).sum()
    hd.delta_attention_step(*(x[:, 0].detach() if x.dim() > 1 else x for x in ins[:5]), state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward()
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(ins[0].detach(), torch.ones_like(ins[0]))
        with pytest.raises(Exception):
            hd.delta_attention(dual, *[x.detach() for x in ins[1:]])


def test_results_do_not_change_from_run_to_run(hd):
    for shape in ((2, 300, 4, 2, 2, 4, 64, 64), (5, 130, 16, 8, 8, 16, 128, 128)):
        ins = [x.requires_grad_() for x in make(*shape, BF16, "token", True, seed=1)]
        d_o = torch.randn(*shape[:3], shape[7], device=DEV).to(BF16)
        runs = []
        for _ in range(3):
            o, s = hd.delta_attention(*ins)
            runs.append([o, s, *torch.autograd.grad(o, ins, d_o)])
        assert all(torch.equal(a, b) for run in runs[1:] for a, b in zip(run, runs[0]))
