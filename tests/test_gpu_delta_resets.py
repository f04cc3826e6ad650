"""The delta rule where log decays are -inf: gradients over sequences that forget their state in the middle of chunks (packed
sequences), and states that hold what is not a number where the first token or a later one forgets them."""
import pytest
import torch

from test_gpu_delta import BF16, DEV, F32, MANY, SHAPES, gradients, hd, make  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("state", [False, True])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] * s[2] < 40] + MANY, ids=str)
def test_gradients_over_resets(hd, shape, state, dtype):  # noqa: F811
    ins = [x.requires_grad_() if x is not None else None for x in make(*shape, dtype, "reset", state, seed=13 + sum(shape))]
    gradients(hd, ins, 0.25, state, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("places", [(0,), (63,), (64,), (0, 1, 2), (62, 63, 64, 65), (31, 32, 96, 129)], ids=str)
@pytest.mark.parametrize("shape", [(2, 130, 2, 1, 2, 2, 64, 64), (1, 130, 1, 1, 1, 1, 200, 64), (5, 130, 16, 16, 16, 16, 128, 128)], ids=str)
def test_resets_at_the_edges_of_chunks(hd, shape, places, dtype):  # noqa: F811
    ins = list(make(*shape, dtype, "token", True, seed=3))
    ins[3][:, list(places)] = -float("inf")
    gradients(hd, [x.requires_grad_() for x in ins], 0.25, True, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("shape", [(2, 100, 2, 2, 2, 2, 64, 64), (2, 40, 2, 2, 2, 2, 256, 64), (5, 100, 16, 16, 16, 16, 64, 128)], ids=str)
def test_a_state_that_the_first_token_forgets(hd, shape, what, dtype):  # noqa: F811
    """Outputs, the last state and every gradient are those of any other state there."""
    ins = list(make(*shape, dtype, "token", True, seed=8))
    ins[3][:, 0] = -float("inf")
    d_o = torch.randn(*shape[:3], shape[7], device=DEV).to(dtype)
    runs = []
    for value in (0.0, what):
        ins[5] = torch.full_like(ins[5], value)
        leaves = [x.detach().requires_grad_() for x in ins]
        o, s = hd.delta_attention(*leaves)
        runs.append([o.detach(), s.detach(), *torch.autograd.grad([o, s], leaves, [d_o, torch.ones_like(s)])])
    assert all(torch.isfinite(x).all() for x in runs[0])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("at", [1, 15, 37, 63, 64, 70])
@pytest.mark.parametrize("shape", [(2, 100, 2, 2, 2, 2, 64, 64), (1, 100, 2, 2, 2, 2, 256, 64), (5, 100, 16, 16, 16, 16, 64, 128)], ids=str)
def test_a_state_that_a_later_token_forgets(hd, shape, at, what, dtype):  # noqa: F811
    """Packed sequences behind one whose state is not a number: from the token that forgets it on, all is as with any other state."""
    ins = list(make(*shape, dtype, "token", True, seed=8))
    ins[3][:, at] = -float("inf")
    d_o = torch.randn(*shape[:3], shape[7], device=DEV).to(dtype)
    runs = []
    for value in (0.0, what):
        ins[5] = torch.full_like(ins[5], value)
        leaves = [x.detach().requires_grad_() for x in ins]
        o, s = hd.delta_attention(*leaves)
        runs.append([s.detach(), *(x[:, at:] for x in (o.detach(), *torch.autograd.grad([o, s], leaves[:5], [d_o, torch.ones_like(s)])))])
        assert value == 0.0 or not torch.isfinite(o[:, :at]).any()
    assert all(torch.isfinite(x).all() for x in runs[0])
    for a, b, n in zip(*runs, ("state", "o", "dq", "dk", "dv", "dlog_a", "dbeta")):
        assert torch.equal(a, b), n
