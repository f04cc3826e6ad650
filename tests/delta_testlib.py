"""The delta rule with a decay in plain float64, token by token from the definition (its gradients by autograd), and beam search's
selection over sorted candidates.

Tolerances of attention_testlib, for the same reasons: float32 results are sums whose operands count with 24 bits, in at most 256
products each before they are joined (256 roundings of 2^-24 are 1.5e-5); a bfloat16 result is rounded once itself (at most 2^-8 of an
element, which is below 2^-9 in the 2-norm) and hangs on at most two operands that are.  The recurrence does not enlarge what is off as long as beta |k|^2 lies between 0 and 2 and
decays between 0 and 1: (I - beta k k^T) has no singular value above one."""
import torch

from attention_testlib import heads


def delta64(q, k, v, log_a, beta, state0=None, scale=1.0, lengths=None):
    """(o, state) of S_t = a_t S_{t-1} + beta_t k_t (v_t - a_t S_{t-1}^T k_t)^T, o_t = scale S_t^T q_t, one token at a time."""
    b, t = q.shape[:2]
    h = log_a.shape[-1]
    q, k, v = (heads(x.double(), h) for x in (q, k, v))
    a, beta = log_a.double().expand(b, t, h), beta.double()
    s = torch.zeros(b, h, q.shape[-1], v.shape[-1], dtype=torch.float64, device=q.device) if state0 is None else state0.double()
    live = torch.full((b,), t, device=q.device) if lengths is None else lengths.long().clamp(0, t)
    outs = []
    for i in range(t):
        now = i < live
        decay = a[:, i].exp()[..., None, None]
        old = torch.where(decay == 0, 0.0, decay * s)  # a decay of exactly zero forgets the state
        error = v[:, i] - (k[:, i].unsqueeze(-2) @ old).squeeze(-2)
        new = old + k[:, i].unsqueeze(-1) * (beta[:, i, :, None] * error).unsqueeze(-2)
        s = torch.where(now[:, None, None, None], new, s)
        o = scale * (q[:, i].unsqueeze(-2) @ s).squeeze(-2)
        outs.append(torch.where(now[:, None, None], o, 0.0))
    o = torch.stack(outs, 1) if outs else q[..., :1].expand(b, 0, h, v.shape[-1])
    return o, s


def select64(logits, scores, keep, ended=None, end_token=0):
    """(scores, parents, tokens) of the best continuations: all candidates sorted, equal ones in the order of their places."""
    b, w, n = logits.shape
    x = logits.double()
    total = torch.logsumexp(x, -1, keepdim=True)
    x = x - total + scores.double()[..., None]
    out = ~(torch.isfinite(total) & torch.isfinite(scores)[..., None])
    x = torch.where(out | ~torch.isfinite(logits), -float("inf"), x)
    if ended is not None:
        stays = torch.full_like(x, -float("inf"))
        stays[..., end_token] = torch.where(torch.isfinite(scores), scores.double(), -float("inf"))
        x = torch.where(ended.bool()[..., None], stays, x)
    best, at = torch.sort(x.flatten(1), dim=-1, descending=True, stable=True)
    return best[:, :keep], at[:, :keep] // n, at[:, :keep] % n
