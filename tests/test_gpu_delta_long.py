"""The delta rule over many chunks of many sequences at once: the passes on tcgen05 go through all of their barriers many times, and
every CTA that takes chunk after chunk takes several.  Against the float64 form, and bit for bit from run to run.

Tolerances of attention_testlib.  They hold for any number of tokens: with beta |k|^2 between 0 and 2 and decays up to 1 nothing that
is off grows, and decays of 0.73 to 0.999 forget what is off within a few hundred tokens."""
import pytest
import torch

from attention_testlib import close, leaf64
from delta_testlib import delta64
from test_gpu_delta import BF16, DEV, NAMES, hd, make  # noqa: F401

pytestmark = pytest.mark.gpu

# (batch, tokens, heads, q, k and v heads, key and value width): eleven chunks of 80 pairs, 880 of them for 148 CTAs
SHAPES = [(5, 700, 16, 16, 16, 16, 64, 128), (5, 650, 16, 8, 8, 16, 128, 104)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_many_chunks_of_many_sequences(hd, shape):  # noqa: F811
    ins = [x.requires_grad_() for x in make(*shape, BF16, "token", True, seed=11)]
    d_o = torch.randn(*shape[:3], shape[7], device=DEV).to(BF16)
    d_s = torch.randn(shape[0], shape[2], shape[6], shape[7], device=DEV)
    runs = []
    for _ in range(4):
        o, s = hd.delta_attention(*ins)
        runs.append([o.detach(), s.detach(), *torch.autograd.grad([o, s], ins, [d_o, d_s])])
    hd.check(DEV)
    assert all(torch.equal(a, b) for run in runs[1:] for a, b in zip(run, runs[0]))
    o, s, *grads = runs[0]
    del runs
    wide = [leaf64(x) for x in ins]
    want_o, want_s = delta64(*wide, scale=shape[6] ** -0.5)
    close(o, want_o, "o")
    close(s, want_s, "state")
    for a, b, n in zip(grads, torch.autograd.grad([want_o, want_s], wide, [d_o.double(), d_s.double()]), NAMES):
        close(a, b, n)
