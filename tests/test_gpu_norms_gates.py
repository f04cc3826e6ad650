"""gated_norm in float32 element by element over the whole range of gates, where the logistic function itself is tiny."""
import pytest
import torch

from attention_testlib import gated_norm64, leaf64
from test_gpu_norms import DEV, F32, ha  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [4, 3])
def test_every_element_is_good_to_a_few_roundings(ha, d):  # noqa: F811
    """A row of d <= 4: exponential 2 (an ulp is two roundings), its sum with 1 and the quotient 2, four squares, their sum, mean and
    eps 5, the root 4, half of the sum's share of them at least, and five products: below 24 roundings of 2^-24.  The gate's
    gradient is d n w s (1 + z (1 - s)): of the size of what it is added up from."""
    n = 4001
    g = torch.Generator(device=DEV).manual_seed(d)
    z = torch.linspace(-80, 80, n * d, device=DEV)[torch.randperm(n * d, device=DEV, generator=g)].view(n, d)
    x, w, dy = (torch.randn(*s, device=DEV, generator=g) for s in ((n, d), (d,), (n, d)))
    ins, wide = [t.requires_grad_() for t in (x, z, w)], [leaf64(t) for t in (x, z, w)]
    y, want = ha.gated_norm(*ins), gated_norm64(*wide)
    tol = 24 * 2.0 ** -24
    assert y.dtype == F32
    off = (y.detach().double() - want.detach()).abs() / want.detach().abs()
    assert float(off.max()) <= tol, f"y: {float(off.max()) / tol:.3g} times the tolerance at a gate of {float(z.detach().flatten()[off.argmax()]):.3g}"
    got, = torch.autograd.grad(y, z, dy)
    back, = torch.autograd.grad(want, wide[1], dy.double())
    z64 = wide[1].detach()
    size = (want.detach() * dy.double()).abs() * (1 + z64.abs()) / z64.abs()
    off = (got.double() - back).abs() / size
    assert float(off.max()) <= 2 * tol, f"dgate: {float(off.max()) / tol:.3g} times the tolerance"
