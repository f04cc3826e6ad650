"""The operators together, as the example model has them: gradients of a whole model, training, a prompt continued by steps."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decay_model", os.path.join(ROOT, "examples", "decay_model.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def build(example, dtype, dim=128, heads=4, seed=3):
    torch.manual_seed(seed)
    return example.Model(50, dim, 2, heads, dtype).cuda()


@pytest.mark.parametrize("tokens", [1, 2, 7, 150])
def test_steps_continue_a_prompt(example, tokens):
    # float32 throughout: both ways compute the same sums in another order, some thousands of roundings of 2^-24 in all
    model = build(example, torch.float32)
    t = torch.randint(50, (3, tokens + 5), device="cuda")
    with torch.no_grad():
        want, last = model(t)
        logits, states = model(t[:, :tokens])
        torch.testing.assert_close(logits[:, -1], want[:, tokens - 1], rtol=1e-3, atol=1e-3)
        for i in range(5):
            logits, states = model(t[:, tokens + i], states)
            torch.testing.assert_close(logits, want[:, tokens + i], rtol=1e-3, atol=1e-3)
    for a, b in zip(states, last):
        torch.testing.assert_close(a, b, rtol=1e-3, atol=1e-3)


def test_gradients_against_differences(example):
    # the loss along one direction of all parameters; h ~ eps^(1/3) of float32 makes its error and the difference's about 1e-2
    model = build(example, torch.float32, dim=64, heads=2)
    t = torch.randint(50, (2, 45), device="cuda")

    def loss():
        logits, _ = model(t[:, :-1])
        return torch.nn.functional.cross_entropy(logits.double().flatten(0, 1), t[:, 1:].flatten())

    model.zero_grad(set_to_none=True)
    loss().backward()
    grads = [p.grad for p in model.parameters()]
    size = torch.stack([g.double().pow(2).sum() for g in grads]).sum().sqrt()
    direction = [(g.double() / size) for g in grads]  # the gradient's own: the difference is its length
    h = 1e-2
    with torch.no_grad():
        start = [p.clone() for p in model.parameters()]
        ends = []
        for sign in (1, -1):
            for p, s, d in zip(model.parameters(), start, direction):
                p.copy_(s + sign * h * d)
            ends.append(float(loss()))
    assert abs((ends[0] - ends[1]) / (2 * h) / float(size) - 1) < 2e-2


def test_gradients_with_saved_tensors_on_the_host(example):
    model = build(example, torch.float32, dim=64, heads=2)
    t = torch.randint(50, (2, 33), device="cuda")

    def grads():
        model.zero_grad(set_to_none=True)
        model(t)[0].sum().backward()
        return [p.grad.clone() for p in model.parameters()]

    want = grads()
    with torch.autograd.graph.save_on_cpu():
        model.zero_grad(set_to_none=True)
        total = model(t)[0].sum()
        junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]  # where freed tensors were
        total.backward()
    del junk
    for a, p in zip(want, model.parameters()):
        assert torch.equal(a, p.grad)


def test_training_lowers_the_loss(example):
    model = build(example, torch.bfloat16)
    losses = example.train(model, 40, 16, 64)
    assert all(x == x for x in losses)
    assert sum(losses[-5:]) < 0.9 * sum(losses[:5])


def test_generate_runs_one_pass_and_steps(example):
    model = build(example, torch.bfloat16)
    prompt = torch.randint(50, (5, 19), device="cuda")
    made = example.generate(model, prompt, 6)
    assert made.shape == (5, 6) and int(made.min()) >= 0 and int(made.max()) < 50
    assert torch.equal(made, example.generate(model, prompt, 6))
