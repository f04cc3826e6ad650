"""The delta rule and the search together, as the example model has them: gradients of a whole model, training that runs, a prompt
continued by steps, a search whose scores are the model's own."""
import pytest
import torch

from test_gpu_decay_model import example  # noqa: F401

pytestmark = pytest.mark.gpu


def build(example, dtype, dim=128, heads=4, seed=3):  # noqa: F811
    torch.manual_seed(seed)
    return example.Model(50, dim, 2, heads, dtype, delta=True).cuda()


@pytest.mark.parametrize("tokens", [1, 2, 7, 150])
def test_steps_continue_a_prompt(example, tokens):  # noqa: F811
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


def test_gradients_against_differences(example):  # noqa: F811
    # the loss along the gradient of all parameters; h ~ eps^(1/3) of float32 makes its error and the difference's about 1e-2
    model = build(example, torch.float32, dim=64, heads=2)
    t = torch.randint(50, (2, 45), device="cuda")

    def loss():
        logits, _ = model(t[:, :-1])
        return torch.nn.functional.cross_entropy(logits.double().flatten(0, 1), t[:, 1:].flatten())

    loss().backward()
    grads = [p.grad.double() for p in model.parameters()]
    size = torch.stack([g.pow(2).sum() for g in grads]).sum().sqrt()
    h, ends = 1e-2, []
    with torch.no_grad():
        start = [p.clone() for p in model.parameters()]
        for sign in (1, -1):
            for p, s, g in zip(model.parameters(), start, grads):
                p.copy_((s.double() + sign * h * g / size).float())
            ends.append(loss())
    assert abs(float((ends[0] - ends[1]) / (2 * h) / size) - 1) < 2e-2


def test_training_and_a_search_run(example):  # noqa: F811
    model = build(example, torch.bfloat16)
    losses = example.train(model, 3, 4, 70)
    assert len(losses) == 3 and all(x == x for x in losses)
    prompt = torch.randint(50, (3, 40), device="cuda")
    made, scores = example.search(model, prompt, 6, 4)
    assert made.shape == (3, 4, 6) and (scores[:, :-1] >= scores[:, 1:]).all()


@pytest.mark.parametrize("beams", [1, 3, 8])
def test_scores_of_a_search_are_the_models(example, beams):  # noqa: F811
    """The log probability of every continuation found, from one pass over prompt and continuation: five tokens' worth of float32 sums."""
    model = build(example, torch.float32)
    prompt = torch.randint(50, (2, 33), device="cuda")
    made, scores = example.search(model, prompt, 5, beams)
    with torch.no_grad():
        whole = torch.cat([prompt[:, None].expand(-1, beams, -1), made], -1)
        logits, _ = model(whole.flatten(0, 1)[:, :-1])
        taken = torch.log_softmax(logits[:, 32:].double(), -1).gather(-1, made.flatten(0, 1)[..., None]).sum((1, 2))
    torch.testing.assert_close(scores.double().flatten(), taken, rtol=1e-3, atol=1e-3)
    assert len({tuple(x) for x in made[0].tolist()}) == beams
    if beams == 1:
        assert torch.equal(made[:, 0], example.generate(model, prompt, 5))
