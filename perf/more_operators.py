"""Workloads of the delta rule with a decay (whole sequences, training, single tokens) and of beam search over models
whose memory is a pool of states.

Two sides compute the same operators: elementary torch operations in 32 bits, or 64 where choices hang on them (`own`
false), and the package's kernels (`own` true).  The operators:

* prompt:  o_t = scale * S_t^T q_t with S_t = a_t S_{t-1} + beta_t k_t (v_t - a_t S_{t-1}^T k_t)^T, a_t = exp(log_a_t), over
           whole prompts;
* train:   the same with the gradients of every input;
* step:    one token of it for each sequence, the states updated in place;
* select:  the best continuations of every group of beams by score + log_softmax(logits);
* reorder: every beam's state becomes that of its parent, in place.
"""
import math

import torch

own = False
CHUNK = 64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases

def delta_case(kind, b, t, h, hk, kd, vd, dtype, decay, state, ragged):
    """h heads of values, decays and states; hk of queries and keys."""
    return {"kind": kind, "b": b, "t": t, "h": h, "hk": hk, "kd": kd, "vd": vd, "dtype": dtype, "decay": decay, "state": state,
            "ragged": ragged}


def listed():
    return [
        # a short question to a small model: the cost of a call
        {"name": "prompt_short", **delta_case("prompt", 1, 17, 4, 4, 64, 64, "bf16", "token", False, False)},
        # a batch of ordinary prompts in the widths of a model of 2048 channels
        {"name": "prompt_batch", **delta_case("prompt", 4, 2048, 16, 16, 128, 128, "bf16", "token", False, False)},
        # one long document of odd length, continued from a kept state, with a fixed decay for each head
        {"name": "prompt_long", **delta_case("prompt", 1, 16385, 8, 8, 128, 128, "bf16", "head", True, False)},
        # prompts of different lengths, queries and keys shared by two heads, in 32 bits
        {"name": "prompt_ragged_f32", **delta_case("prompt", 3, 1000, 8, 4, 64, 64, "f32", "token", True, True)},
        # the training step of the 2048-channel model
        {"name": "train_batch", **delta_case("train", 8, 2048, 16, 16, 128, 128, "bf16", "token", False, False)},
        # training with shared queries and keys, odd length, a width that no tile divides, states carried over segments
        {"name": "train_shared", **delta_case("train", 3, 517, 8, 4, 96, 64, "bf16", "token", True, False)},
        # the next token for one user
        {"name": "step_one", "kind": "step", "b": 1, "h": 16, "hk": 16, "kd": 128, "vd": 128, "dtype": "bf16", "pool": 4},
        # the next token for a large batch of users, whose states lie scattered in a pool
        {"name": "step_many", "kind": "step", "b": 256, "h": 16, "hk": 16, "kd": 128, "vd": 128, "dtype": "bf16", "pool": 300},
        # one user's four beams over a small vocabulary
        {"name": "select_one", "kind": "select", "b": 1, "w": 4, "n": 32000, "k": 4, "dtype": "bf16", "ended": False},
        # a batch of searches, eight beams each, some of them ended, over a large vocabulary of odd size, logits in 32 bits
        {"name": "select_many", "kind": "select", "b": 32, "w": 8, "n": 100003, "k": 8, "dtype": "f32", "ended": True},
        # the states of one user's four beams
        {"name": "reorder_one", "kind": "reorder", "b": 1, "w": 4, "h": 16, "kd": 128, "vd": 128, "pool": 6},
        # the states of 48 searches of four beams, scattered in a pool
        {"name": "reorder_many", "kind": "reorder", "b": 48, "w": 4, "h": 16, "kd": 128, "vd": 128, "pool": 200},
    ]


def between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "train", "train", "step", "select", "select", "reorder"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    small = 8 if dtype == "f32" else 1
    if kind in ("prompt", "train"):
        h = rng.choice([4, 8, 12, 16, 24])
        most = (130000 if kind == "prompt" else 200000) // small  # tokens times heads
        t = between(rng, 2, min(8192, most // h))
        b = between(rng, 1, max(1, min(32, most // (h * t))))
        return delta_case(kind, b, t, h, rng.choice([h, h, h // 2, h // 4]), rng.choice([64, 96, 128, 128]),
                          rng.choice([64, 80, 128, 128]), dtype, rng.choice(["token", "token", "head"]), rng.random() < 0.5,
                          rng.random() < 0.25)
    if kind == "step":
        h = rng.choice([4, 8, 16, 24])
        b = between(rng, 1, 160)
        return {"kind": "step", "b": b, "h": h, "hk": rng.choice([h, h // 2, h // 4]), "kd": rng.choice([64, 96, 128]),
                "vd": rng.choice([64, 80, 128]), "dtype": dtype, "pool": b + rng.randrange(40)}
    if kind == "select":
        w = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
        n = between(rng, 1000, 150000)
        return {"kind": "select", "b": between(rng, 1, max(1, min(64, 24000000 // (w * n)))), "w": w, "n": n,
                "k": rng.choice([w, w, 2 * w]), "dtype": dtype, "ended": rng.random() < 0.5}
    b, w = between(rng, 1, 40), rng.choice([2, 3, 4, 4])
    return {"kind": "reorder", "b": b, "w": w, "h": rng.choice([4, 8, 16]), "kd": rng.choice([64, 96, 128]),
            "vd": rng.choice([64, 80, 128]), "pool": b * w + rng.randrange(20)}


# --------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case.get("dtype", "f32")]

    def normal(*shape, to=dt, spread=1.0, about=0.0):
        return torch.randn(*shape, device="cuda", generator=g).mul_(spread).add_(about).to(to)

    def unit(*shape):  # queries and keys of a layer of this kind have length one
        x = normal(*shape, to=torch.float32)
        return (x / x.norm(dim=-1, keepdim=True)).to(dt)

    s = {"case": case}
    if case["kind"] in ("prompt", "train"):
        b, t, h, hk, kd, vd = (case[n] for n in ("b", "t", "h", "hk", "kd", "vd"))
        s["q"], s["k"], s["v"] = unit(b, t, hk, kd), unit(b, t, hk, kd), normal(b, t, h, vd)
        s["beta"] = torch.sigmoid(normal(b, t, h, to=torch.float32))
        if case["decay"] == "token":  # the gate of a linear recurrence: logsigmoid of a normal
            s["log_a"] = torch.nn.functional.logsigmoid(normal(b, t, h, to=torch.float32, about=3.0))
        else:  # windows of about 2**4 to 2**10 tokens
            window = 4 + 6 * torch.arange(h, device="cuda") / max(1, h - 1) + normal(h, to=torch.float32, spread=0.1)
            s["log_a"] = torch.log1p(-torch.exp2(-window))
        s["state0"] = normal(b, h, kd, vd, to=torch.float32) if case["state"] else None
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(0, t + 1, (b,), device="cuda", generator=g, dtype=torch.int32)
        if case["kind"] == "train":
            s["do"] = normal(b, t, h, vd)
            s["dstate"] = normal(b, h, kd, vd, to=torch.float32) if case["state"] else None
            for n in ("q", "k", "v", "log_a", "beta", "state0"):
                if s[n] is not None:
                    s[n].requires_grad_()
    elif case["kind"] == "step":
        b, h, hk, kd, vd = (case[n] for n in ("b", "h", "hk", "kd", "vd"))
        s["q"], s["k"], s["v"] = unit(b, hk, kd), unit(b, hk, kd), normal(b, h, vd)
        s["beta"] = torch.sigmoid(normal(b, h, to=torch.float32))
        s["log_a"] = torch.nn.functional.logsigmoid(normal(b, h, to=torch.float32, about=3.0))
        s["state"] = normal(case["pool"], h, kd, vd, to=torch.float32)
        s["slots"] = torch.randperm(case["pool"], device="cuda", generator=g)[:b].to(torch.int32)
    elif case["kind"] == "select":
        b, w, n = case["b"], case["w"], case["n"]
        s["logits"] = normal(b, w, n, spread=3.0)
        s["scores"] = normal(b, w, to=torch.float32, spread=2.0, about=-12.0).sort(-1, descending=True).values
        s["end"] = n // 3
        s["ended"] = torch.rand(b, w, device="cuda", generator=g) < 0.2 if case["ended"] else None
    else:
        b, w = case["b"], case["w"]
        s["state"] = normal(case["pool"], case["h"], case["kd"], case["vd"], to=torch.float32)
        s["slots"] = torch.randperm(case["pool"], device="cuda", generator=g)[:b * w].to(torch.int32).view(b, w)
        s["parents"] = torch.randint(0, w, (b, w), device="cuda", generator=g, dtype=torch.int32)
    return s


# ---------------------------------------------------------------------------------------- plain forms

def to_heads(x, h):
    """[..., heads, width] -> [..., h, width]: every head of x serves h / heads neighbours."""
    n = x.shape[-2]
    return x if n == h else x.unsqueeze(-2).expand(*x.shape[:-1], h // n, x.shape[-1]).reshape(*x.shape[:-2], h, x.shape[-1])


def sums_between(x):
    """y[i, j] = x[j + 1] + ... + x[i] for j <= i, else -inf, without cancellation."""
    n = x.shape[-1]
    at = torch.arange(n, device=x.device)
    y = x.unsqueeze(-1).expand(*x.shape, n).masked_fill(at[:, None] <= at[None, :], 0.0).cumsum(-2)
    return y.masked_fill(at[:, None] < at[None, :], -math.inf)


def inverse_from(m):
    """(I + m)^-1 of strictly lower m [.., n, n], n a power of two, from blocks of one upwards: with A and D inverted,
    the inverse of [[A, 0], [B, D]] has -D^-1 B A^-1 below the diagonal."""
    n = m.shape[-1]
    at = torch.arange(n, device=m.device)
    x = torch.eye(n, device=m.device, dtype=m.dtype)
    size = 1
    while size < n:
        joins = (at[:, None] // (2 * size) == at[None, :] // (2 * size)) & (at[:, None] // size > at[None, :] // size)
        x = x - x @ (m * joins) @ x
        size *= 2
    return x


def plain_delta(q, k, v, log_a, beta, state0, scale, lengths):
    """In chunks: within one the tokens' writes solve a triangular system, and only the states go from one to the next."""
    b, t = q.shape[:2]
    h = log_a.shape[-1]
    dt = q.dtype
    q, k, v = (to_heads(x.float(), h) for x in (q, k, v))
    a = log_a.float().expand(b, t, h)
    beta = beta.float()
    if lengths is not None:
        live = (torch.arange(t, device=q.device) < lengths[:, None])[..., None]
        k, v, a, beta = k * live[..., None], v * live[..., None], a * live, beta * live
    n = -(-t // CHUNK)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, n * CHUNK - t)).unflatten(1, (n, CHUNK))  # noqa: E731
    q, k, v = (cut(x).permute(0, 3, 1, 2, 4) for x in (q, k, v))  # [b, h, n, chunk, width]
    a, beta = (cut(x).permute(0, 3, 1, 2) for x in (a, beta))
    c = a.cumsum(-1)
    between_tokens = sums_between(a).exp()
    inverse = inverse_from(((k @ k.transpose(-1, -2)) * between_tokens * beta[..., None]).tril(-1))
    early = c.exp()[..., None]
    writes = inverse @ (v * beta[..., None])
    reads = inverse @ (k * beta[..., None] * early)
    near = (q @ k.transpose(-1, -2)) * between_tokens
    late = (k * (c[..., -1:] - c).exp()[..., None]).transpose(-1, -2)
    q = q * early
    state = torch.zeros(b, h, q.shape[-1], v.shape[-1], device=q.device) if state0 is None else state0.float()
    outs = []
    for i in range(n):
        new = writes[:, :, i] - reads[:, :, i] @ state
        outs.append(q[:, :, i] @ state + near[:, :, i] @ new)
        state = state * early[:, :, i, -1:] + late[:, :, i] @ new
    o = (torch.stack(outs, 2) * scale).permute(0, 2, 3, 1, 4).flatten(1, 2)[:, :t]
    if lengths is not None:
        o = o * live[..., None]
    return o.to(dt), state


def plain_step(q, k, v, log_a, beta, state, scale, slots):
    h = log_a.shape[-1]
    at = slots.long()
    k, v, qf = (to_heads(x.float(), h) for x in (k, v, q))
    new = state[at] * log_a.exp()[..., None, None]
    error = (v - (k.unsqueeze(-2) @ new).squeeze(-2)) * beta[..., None]
    new = new + k.unsqueeze(-1) * error.unsqueeze(-2)
    state[at] = new
    return ((qf * scale).unsqueeze(-2) @ new).squeeze(-2).to(q.dtype)


def plain_select(logits, scores, k, ended, end):
    """In 64 bits: which of two near candidates is taken hangs on their difference."""
    b, w, n = logits.shape
    x = logits.double()
    top = x.amax(-1, keepdim=True)
    x = x - (top + (x - top).exp().sum(-1, keepdim=True).log()) + scores.double()[..., None]
    if ended is not None:
        only = torch.arange(n, device=x.device) == end
        x = torch.where(ended[..., None], torch.where(only, scores.double()[..., None], -math.inf), x)
    x = x.flatten(1)
    # the k-th best value, and of its equals as many as are wanted, the first ones
    least = x.topk(k, dim=-1).values[:, -1:]
    above, equal = x > least, x == least
    taken = above | (equal & (equal.cumsum(-1) <= k - above.sum(-1, keepdim=True)))
    total = w * n
    at = total - torch.where(taken, total - torch.arange(total, device=x.device), 0).topk(k, dim=-1).values  # in order of place
    values, order = x.gather(1, at).sort(dim=-1, descending=True, stable=True)
    at = at.gather(1, order)
    return values.float(), (at // n).int(), (at % n).int()


def plain_reorder(state, parents, slots):
    state[slots.long()] = state[slots.gather(1, parents.long()).long()]


# ------------------------------------------------------------------------------------------- the pass

def gradients(outputs, grads, inputs):
    names = [n for n, x in inputs.items() if x is not None]
    pairs = [(o, g) for o, g in zip(outputs, grads) if g is not None]
    got = torch.autograd.grad([o for o, _ in pairs], [inputs[n] for n in names], [g for _, g in pairs])
    return {"d" + n: g for n, g in zip(names, got)}


def run(s):
    case = s["case"]
    if own:
        from paper_2311_06281_b200 import heinsen_beam as hb
        from paper_2311_06281_b200 import heinsen_delta as hd
    if case["kind"] in ("prompt", "train"):
        scale = case["kd"] ** -0.5
        if own:
            o, state = hd.delta_attention(s["q"], s["k"], s["v"], s["log_a"], s["beta"], s["state0"], scale=scale, lengths=s["lengths"])
        else:
            o, state = plain_delta(s["q"], s["k"], s["v"], s["log_a"], s["beta"], s["state0"], scale, s["lengths"])
        out = {"o": o, "state": state}
        if case["kind"] == "train":
            out.update(gradients([o, state], [s["do"], s["dstate"]], {n: s[n] for n in ("q", "k", "v", "log_a", "beta", "state0")}))
        return out
    if case["kind"] == "step":
        call = hd.delta_attention_step if own else plain_step
        o = call(s["q"], s["k"], s["v"], s["log_a"], s["beta"], s["state"], scale=case["kd"] ** -0.5, slots=s["slots"])
        return {"o": o, "state": s["state"]}
    if case["kind"] == "select":
        if own:
            scores, parents, tokens = hb.beam_select(s["logits"], s["scores"], case["k"], ended=s["ended"], end_token=s["end"])
        else:
            scores, parents, tokens = plain_select(s["logits"], s["scores"], case["k"], s["ended"], s["end"])
        return {"scores": scores, "parents": parents, "tokens": tokens}
    if own:
        hb.beam_reorder(s["state"], s["parents"], slots=s["slots"])
    else:
        plain_reorder(s["state"], s["parents"], s["slots"])
    return {"state": s["state"]}


def work(case):
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] in ("prompt", "train"):
        b, t, h, hk, kd, vd = (case[n] for n in ("b", "t", "h", "hk", "kd", "vd"))
        qkv = b * t * (2 * hk * kd + h * vd) * size
        gates = b * t * h * 4 + (b * t * h * 4 if case["decay"] == "token" else h * 4)
        state = b * h * kd * vd * 4
        flops = 6 * b * t * h * kd * vd  # the prediction, the update and the readout of the recurrent form
        moved = qkv + gates + b * t * h * vd * size + state * (2 if case["state"] else 1)
        if case["kind"] == "train":  # dO in, gradients out
            moved += qkv + gates + b * t * h * vd * size + (2 * state if case["state"] else 0)
            flops *= 3.5
        return {"bytes": moved, "flops": flops}
    if case["kind"] == "step":
        b, h, hk, kd, vd = (case[n] for n in ("b", "h", "hk", "kd", "vd"))
        state = b * h * kd * vd
        return {"bytes": 8 * state + b * (2 * hk * kd + 2 * h * vd) * size + 4 * b * (2 * h + 1), "flops": 7 * state}
    if case["kind"] == "select":
        rows = case["b"] * case["w"]
        return {"bytes": rows * case["n"] * size + 5 * rows + 12 * case["b"] * case["k"], "flops": 4 * rows * case["n"]}
    # of w beams with a parent each at random, (1 - 1 / w) w move, and w - 1 others have (1 - 1 / w)^(w - 1) w rows that nobody asks for
    w, row = case["w"], case["h"] * case["kd"] * case["vd"] * 4
    moved, asked = w - 1, w * (1 - (1 - 1 / w) ** (w - 1))
    return {"bytes": case["b"] * (moved + asked) * row + 8 * case["b"] * w, "flops": 0}


# ------------------------------------------------------------------------------- from the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    d = {n: x.detach().double() if isinstance(x, torch.Tensor) and x.is_floating_point() else x for n, x in s.items()}
    with torch.no_grad():
        return {"prompt": exact_delta, "train": exact_delta, "step": exact_step, "select": exact_select,
                "reorder": exact_reorder}[case["kind"]](case, d)


def exact_delta(case, d):
    """Token by token.  The gradients go back from the last token, with the states before each of KEPT tokens formed again from
    that before the first of them."""
    KEPT = 32
    b, t, h, hk, kd, vd = (case[n] for n in ("b", "t", "h", "hk", "kd", "vd"))
    scale, train = kd ** -0.5, case["kind"] == "train"
    head = torch.arange(h, device="cuda") * hk // h
    q, k, v, beta = d["q"][:, :, head], d["k"][:, :, head], d["v"], d["beta"]
    a = d["log_a"].exp().expand(b, t, h)
    live = torch.ones(b, t, device="cuda", dtype=torch.bool)
    if d["lengths"] is not None:
        live = torch.arange(t, device="cuda") < d["lengths"][:, None]
    state = torch.zeros(b, h, kd, vd, dtype=torch.float64, device="cuda") if d["state0"] is None else d["state0"].clone()

    def decayed(i, s):
        return s * torch.where(live[:, i, None], a[:, i], 1.0)[..., None, None]

    def error(i, s):  # s: decayed
        return v[:, i] - torch.einsum("bhk,bhkv->bhv", k[:, i], s)

    def written(i, s):
        s = decayed(i, s)
        return s + torch.einsum("bhk,bhv->bhkv", k[:, i], error(i, s) * (beta[:, i] * live[:, i, None])[..., None])

    o = torch.zeros(b, t, h, vd, dtype=torch.float64, device="cuda")
    kept = []
    for i in range(t):
        if train and i % KEPT == 0:
            kept.append(state)
        state = written(i, state)
        o[:, i] = torch.einsum("bhk,bhkv->bhv", q[:, i], state) * scale * live[:, i, None, None]
    out = {"o": o, "state": state}
    if not train:
        return out
    ds = torch.zeros_like(state) if d["dstate"] is None else d["dstate"].clone()
    dq, dk, dv, db, da = (torch.zeros_like(x) for x in (q, k, v, beta, beta))
    for n in reversed(range(len(kept))):
        first, last = n * KEPT, min(t, (n + 1) * KEPT)
        states = [kept[n]]
        for i in range(first, last):
            states.append(written(i, states[-1]))
        for i in reversed(range(first, last)):
            on = live[:, i, None]
            do = d["do"][:, i] * on[..., None] * scale
            dq[:, i] = torch.einsum("bhkv,bhv->bhk", states[i + 1 - first], do)
            ds = ds + torch.einsum("bhk,bhv->bhkv", q[:, i], do)
            s, w = decayed(i, states[i - first]), beta[:, i] * on
            e = error(i, s)
            into = torch.einsum("bhk,bhkv->bhv", k[:, i], ds)
            db[:, i] = (into * e).sum(-1) * on
            dv[:, i] = into * w[..., None]
            dk[:, i] = (torch.einsum("bhkv,bhv->bhk", ds, e * w[..., None]) - torch.einsum("bhkv,bhv->bhk", s, dv[:, i])) * on[..., None]
            ds = ds - torch.einsum("bhk,bhv->bhkv", k[:, i], dv[:, i])
            da[:, i] = (ds * s).sum((-1, -2)) * on
            ds = decayed(i, ds)
    shared = lambda x: x.unflatten(2, (hk, h // hk)).sum(3)  # noqa: E731
    out.update({"dq": shared(dq), "dk": shared(dk), "dv": dv, "dbeta": db,
                "dlog_a": da if case["decay"] == "token" else da.sum((0, 1))})
    if d["state0"] is not None:
        out["dstate0"] = ds
    return out


def exact_step(case, d):
    b, h = case["b"], case["h"]
    at = d["slots"].long()
    head = torch.arange(h, device="cuda") * case["hk"] // h
    q, k = d["q"][:, head], d["k"][:, head]
    state = d["state"].clone()
    old = torch.einsum("bh,bhkv->bhkv", d["log_a"].exp(), state[at])
    wrong = d["v"] - torch.einsum("bhk,bhkv->bhv", k, old)
    state[at] = old + torch.einsum("bh,bhk,bhv->bhkv", d["beta"], k, wrong)
    return {"o": torch.einsum("bhk,bhkv->bhv", q, state[at]) * case["kd"] ** -0.5, "state": state}


def exact_select(case, d):
    """Every group by itself: its candidates sorted, equal ones in the order of their places."""
    n, found = case["n"], []
    for i in range(case["b"]):
        rows = torch.log_softmax(d["logits"][i], -1) + d["scores"][i][:, None]
        if d["ended"] is not None:
            stays = torch.full_like(rows, -math.inf)
            stays[:, d["end"]] = d["scores"][i]
            rows = torch.where(d["ended"][i][:, None], stays, rows)
        found.append(torch.sort(rows.reshape(-1), descending=True, stable=True))
    best = torch.stack([f.values[:case["k"]] for f in found])
    at = torch.stack([f.indices[:case["k"]] for f in found])
    return {"scores": best, "parents": torch.div(at, n, rounding_mode="floor"), "tokens": at.remainder(n)}


def exact_reorder(case, d):
    state = d["state"].clone()
    for i in range(case["b"]):
        for j in range(case["w"]):
            state[int(d["slots"][i, j])] = d["state"][int(d["slots"][i, int(d["parents"][i, j])])]
    return {"state": state}
