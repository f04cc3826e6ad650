"""Every element of decay_attention's output and of dq, dk and dv against a bound of its own, from the roundings that are made
on the way to it (a tolerance of the norm lets a single wrong element pass).

All four are one formula, out_i = scale (sum_{j<=i} e^{c_i-c_j} (X_i.Y_j) Z_j + e^{c_i} X_i S) over a chunk, with S the state
before it; dk and dv run from the last token to the first.  With u = 2^-8, half of bfloat16's eps (1 + 2^-8 is rounded to 1):
  bfloat16   the weights e^{c_i-c_j} (X_i.Y_j) and the elements of S are rounded to bfloat16 before their products, the result once
             more: u (1 + u) of the sum of the products' sizes and u of the result (heads that share a tensor: of every summand);
  both       1.5e-5 of the sum with |X_i| |Y_j| in the place of |X_i.Y_j|, for what is computed in float32.
"""
import pytest
import torch

from test_gpu_attention import BF16, DEV, F32, ha, make  # noqa: F401

pytestmark = pytest.mark.gpu


def with_bounds(x, y, z, a, s, scale, chunk):
    """(out, sum of sizes with |X.Y|, with |X||Y|) for [heads, tokens, dim] in 64 bits, decays [heads, tokens], state [heads, dx, dz]."""
    outs = []
    for t0 in range(0, x.shape[1], chunk):
        at = slice(t0, t0 + chunk)
        c = a[:, at].clamp(min=-1e4).cumsum(-1)
        w = scale * torch.exp((c[:, :, None] - c[:, None, :]).tril()).tril()
        early = scale * torch.exp(c)[..., None]
        p, far = w * (x[:, at] @ y[:, at].mT), x[:, at].abs() @ s.abs() * early
        outs.append((p @ z[:, at] + early * (x[:, at] @ s), p.abs() @ z[:, at].abs() + far,
                     (w * (x[:, at].abs() @ y[:, at].abs().mT)) @ z[:, at].abs() + far))
        late = torch.exp(c[:, -1:] - c)[..., None]
        s = torch.exp(c[:, -1])[:, None, None] * s + (y[:, at] * late).mT @ z[:, at]
    return [torch.cat(o, 1) for o in zip(*outs)]


@pytest.mark.parametrize("dtype,chunk", [(BF16, 128), (F32, 32)])
@pytest.mark.parametrize("decay", ["token", "strong", "reset"])
@pytest.mark.parametrize("t,h,kd,vd", [(128, 3, 64, 128), (384, 60, 128, 128), (256, 2, 96, 72), (1280, 2, 128, 64)])
def test_every_element_is_within_the_bound_of_its_roundings(ha, t, h, kd, vd, decay, dtype, chunk):  # noqa: F811
    q, k, v, log_a, s0 = make(1, t, h, h, h, h, kd, vd, dtype, decay, True, seed=t + h)
    g = torch.Generator(device=DEV).manual_seed(12)
    d_o, d_s = torch.randn(1, t, h, vd, device=DEV, generator=g).to(dtype), torch.randn(1, h, kd, vd, device=DEV, generator=g)
    ins, scale = [x.requires_grad_() for x in (q, k, v, log_a, s0)], 0.25
    o, s = ha.decay_attention(*ins, scale=scale)
    dq, dk, dv, _, _ = torch.autograd.grad([o, s], ins, [d_o, d_s])
    q, k, v, d = (x.detach()[0].double().transpose(0, 1) for x in (q, k, v, d_o))
    a, s0, d_s = log_a.detach()[0].double().T, s0.detach()[0].double(), d_s[0].double() / scale
    back = torch.cat([torch.zeros_like(a[:, :1]), a[:, 1:].flip(1)], 1)  # the decay between a token and the one behind it
    turned = lambda *x: [y.flip(1) for y in x]  # noqa: E731
    cases = {"o": (o, with_bounds(q, k, v, a, s0, scale, chunk)), "dq": (dq, with_bounds(d, v, k, a, s0.mT, scale, chunk)),
             "dk": (dk, turned(*with_bounds(*turned(v, d, q), back, d_s.mT, scale, chunk))),
             "dv": (dv, turned(*with_bounds(*turned(k, q, d), back, d_s, scale, chunk)))}
    u = torch.finfo(BF16).eps / 2 if dtype == BF16 else 0.0
    for name, (got, (want, size, whole)) in cases.items():
        bound = u * (1 + u) * size + u * want.abs() + 1.5e-5 * whole
        off = float(((got.detach()[0].double().transpose(0, 1) - want).abs() / bound.clamp(min=2.0 ** -126)).max())
        assert off <= 1, f"{name}: {off:.3g} times the bound of its roundings"
