"""Plain float64 forms of the attention with a decay for each head and of the norms around its block, token by token from
the definition (their gradients by autograd), and the tolerances that the tests compare with.

Tolerances, of the 2-norm of the difference over that of the exact result (`rel`) and of every element over the larger of
its own size and the result's root mean square (`worst`):
  float32 results   rel 1.5e-5: sums of at most 256 products each are accumulated in float32 before they are joined, and
                    256 roundings of 2^-24 are 1.5e-5;
  bfloat16 results  rel 3 * 2^-9: an operand of each of the two products and the result itself are rounded to 8 bits.
A single element may be off by 40 times as much: errors add up over up to a few hundred terms that cancel in it.
Results below the smallest normal float32 number may come out as zero: the kernels flush what lies below it."""
import torch

REL = {torch.float32: 1.5e-5, torch.bfloat16: 3 * 2.0 ** -9}
WORST = 40
TINY = 2.0 ** -126 / 2.0 ** -20  # over the loosest tolerance: a flushed result is within it


def heads(x, h):
    return x.repeat_interleave(h // x.shape[-2], dim=-2)


def attention64(q, k, v, log_a, state0=None, scale=1.0, lengths=None):
    """(o, state) of S_t = exp(log_a_t) S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t, one token at a time."""
    b, t = q.shape[:2]
    h = log_a.shape[-1]
    q, k, v = (heads(x.double(), h) for x in (q, k, v))
    a = log_a.double().expand(b, t, h)
    s = torch.zeros(b, h, q.shape[-1], v.shape[-1], dtype=torch.float64, device=q.device) if state0 is None else state0.double()
    live = torch.full((b,), t, device=q.device) if lengths is None else lengths.long().clamp(0, t)
    outs = []
    for i in range(t):
        now = (i < live)
        decay = torch.where(now[:, None], a[:, i], 0.0).exp()
        # a decay of exactly zero forgets the state
        new = torch.where(decay[..., None, None] == 0, 0.0, decay[..., None, None] * s) + k[:, i].unsqueeze(-1) * v[:, i].unsqueeze(-2)
        s = torch.where(now[:, None, None, None], new, s)
        o = scale * (q[:, i].unsqueeze(-2) @ s).squeeze(-2)
        outs.append(torch.where(now[:, None, None], o, 0.0))
    o = torch.stack(outs, 1) if outs else q[..., :1].expand(b, 0, h, v.shape[-1])
    return o, s


def rms64(x, eps):
    return x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt()


def block_norms64(x, branch, pre, post=None, gate=None, scale=1.0, eps=1e-6):
    x, n, pre = x.double(), branch.double(), pre.double()
    if post is not None:
        n = rms64(n, eps) * post.double()
    r = x + scale * (n if gate is None else gate.double() * n)
    return r, rms64(r, eps) * pre


def gated_norm64(x, gate, weight, eps=1e-6):
    y = rms64(x.double(), eps) * weight.double()
    return y if gate is None else y * gate.double() * torch.sigmoid(gate.double())


def leaf64(t):
    return None if t is None else t.detach().double().requires_grad_()


def close(got, want, what, rel=None):
    """Compares a kernel's tensor with the float64 one at the tolerance of its type."""
    want = want.detach()
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)}, expected {tuple(want.shape)}"
    assert torch.isfinite(got).all(), f"{what}: not finite"
    rel = REL[got.dtype] if rel is None else rel
    if want.numel() == 0:
        return
    d, norm = (got.detach().double() - want), want.norm()
    norm = torch.clamp(norm, min=TINY)
    off = float(d.norm() / norm)
    assert off <= rel, f"{what}: relative error {off:.3g}, tolerance {rel:.3g}"
    rms = float(norm) / want.numel() ** 0.5
    worst = float((d.abs() / torch.clamp(want.abs(), min=rms)).max())
    assert worst <= WORST * rel, f"{what}: worst element {worst:.3g} of the root mean square, tolerance {WORST * rel:.3g}"
