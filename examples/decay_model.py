"""A small language model on the operators of ``paper_2311_06281_b200.heinsen_attention``: training, a prompt, single tokens.

Every layer is: block_norms (the residual sum with the layer before and the norm) -> projections -> decay_attention (whole
sequences; in generation decay_attention_step, one token of every sequence with the states updated in place) -> gated_norm
of every head -> output projection.  With ``delta`` the recurrence is that of ``heinsen_delta``: every token takes out of the state
what it already answers for its key.  The projections are plain matrix products and PyTorch's; the rest is the library's.

    python examples/decay_model.py [--steps 60] [--batch 16] [--tokens 256] [--dim 256] [--layers 2] [--heads 4] [--delta] [--beams 4]

trains on sequences in which one symbol, another for each, stands between random ones and has to be named every time, then
reads a prompt and continues it token by token, the likeliest one each time or, with ``--beams``, by a search over so many
continuations (``heinsen_beam``: the states of a beam become those of its parent).  Needs a GPU.
"""
import argparse
import json
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402
import torch.nn.functional as F  # noqa: E402

from paper_2311_06281_b200 import heinsen_attention as ha  # noqa: E402
from paper_2311_06281_b200 import heinsen_beam as hb  # noqa: E402
from paper_2311_06281_b200 import heinsen_delta as hd  # noqa: E402


class Layer(torch.nn.Module):
    def __init__(self, dim: int, heads: int, delta: bool = False):
        super().__init__()
        self.heads, self.head_dim = heads, dim // heads
        self.norm = torch.nn.Parameter(torch.ones(dim))
        self.project = torch.nn.Parameter(torch.randn(4 * dim, dim) * dim ** -0.5)  # q, k, v and the gate
        self.decay = torch.nn.Parameter(torch.randn(heads, dim) * 0.1 * dim ** -0.5)
        self.decay_bias = torch.nn.Parameter(torch.linspace(-2.0, -7.0, heads))
        self.head_norm = torch.nn.Parameter(torch.ones(self.head_dim))
        self.out = torch.nn.Parameter(torch.randn(dim, dim) * dim ** -0.5)
        self.write = torch.nn.Parameter(torch.randn(heads, dim) * dim ** -0.5) if delta else None  # how much of an error is written

    def forward(self, x, branch, state=None, step=False):
        """The residual stream and what the layer before adds to it, [B, T, dim] (step: [B, dim]); returns the stream, this
        layer's addition and the states, which a step updates in place."""
        x, y = ha.block_norms(x, branch, self.norm)
        q, k, v, gate = F.linear(y, self.project.to(y.dtype)).unflatten(-1, (4, self.heads, self.head_dim)).unbind(-3)
        k = F.normalize(k.float(), dim=-1).to(y.dtype)
        log_a = -F.softplus(F.linear(y.float(), self.decay) + self.decay_bias)
        if self.write is not None:
            beta = torch.sigmoid(F.linear(y.float(), self.write))
            if step:
                o = hd.delta_attention_step(q, k, v, log_a, beta, state)
            else:
                o, state = hd.delta_attention(q, k, v, log_a, beta, state)
        elif step:
            o = ha.decay_attention_step(q, k, v, log_a, state)
        else:
            o, state = ha.decay_attention(q, k, v, log_a, state)
        o = ha.gated_norm(o, gate.contiguous(), self.head_norm)
        return x, F.linear(o.flatten(-2), self.out.to(o.dtype)), state


class Model(torch.nn.Module):
    def __init__(self, vocabulary: int, dim: int, layers: int, heads: int, dtype=torch.bfloat16, delta: bool = False):
        super().__init__()
        self.dtype = dtype
        self.embed = torch.nn.Parameter(torch.randn(vocabulary, dim) * dim ** -0.5)
        self.layers = torch.nn.ModuleList(Layer(dim, heads, delta) for _ in range(layers))
        self.norm = torch.nn.Parameter(torch.ones(dim))

    def forward(self, tokens, states=None):
        """Logits of every token, [B, T, vocabulary] (tokens [B]: of one step, with the states updated), and the states."""
        step = tokens.dim() == 1
        embed = self.embed.to(self.dtype)
        x = F.embedding(tokens, embed) * embed.shape[1] ** 0.5
        branch, left = torch.zeros_like(x), []
        for i, layer in enumerate(self.layers):
            x, branch, state = layer(x, branch, states[i] if states is not None else None, step)
            left.append(state)
        _, y = ha.block_norms(x, branch, self.norm)
        return F.linear(y, embed).float(), left


def sequences(batch: int, tokens: int, vocabulary: int, device, generator) -> torch.Tensor:
    """Random tokens; at even places each sequence's own."""
    t = torch.randint(vocabulary, (batch, tokens), device=device, generator=generator)
    t[:, ::2] = t[:, :1]
    return t


def train(model: Model, steps: int, batch: int, tokens: int, lr: float = 3e-3, seed: int = 0) -> list[float]:
    """The losses of the tokens at even places from the sixth on, one for every step."""
    device, vocabulary = model.embed.device, model.embed.shape[0]
    generator = torch.Generator(device).manual_seed(seed)
    optimizer = torch.optim.AdamW(model.parameters(), lr=lr)
    losses = []
    for _ in range(steps):
        t = sequences(batch, tokens, vocabulary, device, generator)
        logits, _ = model(t[:, :-1])
        loss = F.cross_entropy(logits[:, 5::2].flatten(0, 1), t[:, 6::2].flatten())
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return [float(x) for x in losses]


@torch.no_grad()
def generate(model: Model, prompt: torch.Tensor, count: int) -> torch.Tensor:
    """The `count` likeliest next tokens: the prompt in one pass, then a step for each."""
    logits, states = model(prompt)
    token, tokens = logits[:, -1].argmax(-1), []
    for _ in range(count):
        tokens.append(token)
        logits, states = model(token, states)
        token = logits.argmax(-1)
    return torch.stack(tokens, dim=1)


@torch.no_grad()
def search(model: Model, prompt: torch.Tensor, count: int, beams: int):
    """The `beams` likeliest continuations of `count` tokens that a beam search finds, best first, [B, beams, count], and their log
    probabilities: the prompt in one pass, then for each token a selection, the states moved after their beams, and a step."""
    batch = prompt.shape[0]
    logits, states = model(prompt)
    states = [s.repeat_interleave(beams, 0) for s in states]
    logits = logits[:, -1:].expand(-1, beams, -1)
    scores = torch.full((batch, beams), -float("inf"), device=prompt.device)
    scores[:, 0] = 0.0  # one beam so far
    made = torch.empty(batch, beams, 0, dtype=torch.long, device=prompt.device)
    for i in range(count):
        scores, parents, tokens = hb.beam_select(logits, scores)
        made = torch.cat([made.gather(1, parents.long()[..., None].expand(-1, -1, i)), tokens.long()[..., None]], -1)
        if i + 1 < count:
            for s in states:
                hb.beam_reorder(s, parents)
            logits, states = model(tokens.long().flatten(), states)
            logits = logits.unflatten(0, (batch, beams))
    return made, scores


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("steps", 60), ("batch", 16), ("tokens", 256), ("dim", 256), ("layers", 2), ("heads", 4), ("vocabulary", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--delta", action="store_true")
    ap.add_argument("--beams", type=int, default=0)
    a = ap.parse_args()
    torch.manual_seed(0)
    model = Model(a.vocabulary, a.dim, a.layers, a.heads, delta=a.delta).cuda()
    losses = train(model, a.steps, a.batch, a.tokens)
    t = sequences(a.batch, a.tokens, a.vocabulary, "cuda", torch.Generator("cuda").manual_seed(1))
    prompt, count = t[:, :a.tokens // 2], a.tokens // 2
    made = search(model, prompt, count, a.beams)[0][:, 0] if a.beams else generate(model, prompt, count)
    print(json.dumps({"first_loss": losses[0], "last_loss": losses[-1], "named": float((made == t[:, :1]).float().mean())}))


if __name__ == "__main__":
    main()
