"""Bits that bf16 calls of the delta rule keep between their inputs and their outputs, where sums cancel.

Every number is chosen so that all products and sums are exact in 24 bits: keys that are orthogonal and never meet each other's errors,
decays of one, beta 1, weights 1 + n / 2^11 (n < 256: 12 bits, of which bf16 holds 8), values that are small whole numbers.  A pair of
tokens (columns) has opposite values, so that what is left are the weights' last bits.  A factor of 16 bits or more gives the exact
result, rounded once; one of 8 would give zeros."""
import pytest
import torch

from delta_testlib import delta64
from test_gpu_delta import BF16, DEV, hd  # noqa: F401

pytestmark = pytest.mark.gpu

# few and many (batch, head) pairs: both kinds of pass; keys in chunks of 64 and of 32
SHAPES = [(1, 2, 64, 64), (5, 16, 64, 128), (2, 2, 128, 80), (5, 16, 128, 128), (1, 2, 256, 64)]


def fine(*shape):
    """n / 2^11 with n < 256"""
    return torch.randint(256, shape, device=DEV) * 2.0 ** -11


def whole(*shape):
    return torch.randint(1, 5, shape, device=DEV) * (2.0 * torch.randint(2, shape, device=DEV) - 1)


def orthogonal(b, t, h, kd):
    """Token j has the dimensions 2 j and 2 j + 1: 1 and n / 2^11"""
    k = torch.zeros(b, t, h, kd, device=DEV)
    at = 2 * torch.arange(t, device=DEV)
    k[:, torch.arange(t, device=DEV), :, at] = 1.0
    k[:, torch.arange(t, device=DEV), :, at + 1] = fine(t, b, h)
    return k


@pytest.mark.parametrize("b,h,kd,vd", SHAPES)
def test_what_is_left_of_weights_in_the_output(hd, b, h, kd, vd):  # noqa: F811
    torch.manual_seed(kd + vd)
    t = kd // 2
    k = orthogonal(b, t, h, kd)
    v = whole(b, t // 2, h, vd).repeat_interleave(2, 1)
    v[:, 1::2] *= -1
    ins = [x.to(BF16) for x in (torch.ones(b, t, h, kd, device=DEV), k, v)] + [torch.zeros(h, device=DEV), torch.ones(b, t, h, device=DEV)]
    assert torch.equal(ins[1].float(), k) and torch.equal(ins[2].float(), v)
    o, s = hd.delta_attention(*ins, scale=1.0)
    want_o, want_s = delta64(*ins)
    assert torch.equal(want_o.float().double(), want_o)  # exact in 24 bits
    assert torch.equal(o, want_o.float().to(BF16)) and torch.equal(s.double(), want_s)
    assert (want_o[:, 1::2] != 0).any()
    hd.check(DEV)


@pytest.mark.parametrize("b,h,kd,vd", SHAPES)
def test_what_is_left_of_the_states_gradient_in_dk(hd, b, h, kd, vd):  # noqa: F811
    """The state's gradient lies in dimensions that no key has: dk is its product with the values, and nothing else."""
    torch.manual_seed(kd + vd)
    t = kd // 4
    k = orthogonal(b, t, h, kd)
    v = whole(b, t, h, vd // 2).repeat_interleave(2, -1)
    v[..., 1::2] *= -1
    d_s = torch.zeros(b, h, kd, vd, device=DEV)
    d_s[:, :, kd // 2:] = 1 + fine(b, h, kd // 2, vd)
    ins = [x.to(BF16) for x in (torch.ones(b, t, h, kd, device=DEV), k, v)] + [torch.zeros(h, device=DEV), torch.ones(b, t, h, device=DEV)]
    ins[1].requires_grad_()
    _, s = hd.delta_attention(*ins, scale=1.0)
    (dk,) = torch.autograd.grad(s, ins[1], d_s)
    want = torch.einsum("bthv,bhkv->bthk", v.double(), d_s.double())
    assert torch.equal(want.float().double(), want) and (want != 0).any()
    assert torch.equal(dk, want.float().to(BF16))
    hd.check(DEV)
