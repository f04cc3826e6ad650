"""Workloads of the attention with a decay for each head and of the norms around its block.

Two sides compute the same operators: elementary torch operations in 32 bits (`own` false) and the package's
kernels (`own` true).  The operators:

* prompt: o_t = scale * S_t^T q_t with S_t = exp(log_a_t) S_{t-1} + k_t v_t^T, over whole prompts;
* train:  the same with the gradients of every input;
* step:   one token of it for each sequence, the states updated in place;
* norms:  r = x + scale * gate * rms(branch) * w_post, y = rms(r) * w_pre, alone or with gradients;
* gated:  y = rms(x) * w * silu(gate) over each head, alone or with gradients.
"""
import math

import torch

own = False
EPS = 1e-6
CHUNK = 64
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------- cases

def attention_case(kind, b, t, h, hq, hk, hv, kd, vd, dtype, decay, state, ragged):
    return {"kind": kind, "b": b, "t": t, "h": h, "hq": hq, "hk": hk, "hv": hv, "kd": kd, "vd": vd, "dtype": dtype,
            "decay": decay, "state": state, "ragged": ragged}


def listed():
    return [
        # a short question to a small model: the cost of a call
        {"name": "prompt_short", **attention_case("prompt", 1, 17, 4, 4, 4, 4, 64, 64, "bf16", "token", False, False)},
        # a batch of ordinary prompts in the widths of a model of 2048 channels
        {"name": "prompt_batch", **attention_case("prompt", 4, 2048, 16, 16, 16, 16, 128, 128, "bf16", "token", False, False)},
        # one long document of odd length, continued from a kept state, with a fixed decay for each head
        {"name": "prompt_long", **attention_case("prompt", 1, 65537, 8, 8, 8, 8, 128, 128, "bf16", "head", True, False)},
        # prompts of different lengths, queries and keys shared by the heads, in 32 bits
        {"name": "prompt_ragged_f32", **attention_case("prompt", 3, 1000, 8, 2, 2, 8, 64, 64, "f32", "token", True, True)},
        # the training step of the 2048-channel model
        {"name": "train_batch", **attention_case("train", 8, 2048, 16, 16, 16, 16, 128, 128, "bf16", "token", False, False)},
        # training with grouped keys and values, odd length, a width that no tile divides, states carried over segments
        {"name": "train_grouped", **attention_case("train", 3, 517, 8, 8, 2, 2, 96, 64, "bf16", "token", True, False)},
        # the next token for one user
        {"name": "step_one", "kind": "step", "b": 1, "h": 16, "hq": 16, "hk": 16, "hv": 16, "kd": 128, "vd": 128, "dtype": "bf16", "pool": 4},
        # the next token for a large batch of users, whose states lie scattered in a pool
        {"name": "step_many", "kind": "step", "b": 256, "h": 16, "hq": 16, "hk": 16, "hv": 16, "kd": 128, "vd": 128, "dtype": "bf16", "pool": 300},
        # the norms around the block while tokens are generated
        {"name": "norms_decode", "kind": "norms", "rows": 16, "d": 2048, "dtype": "bf16", "gate": 0, "grad": False},
        # the same in a training step
        {"name": "norms_train", "kind": "norms", "rows": 16384, "d": 2048, "dtype": "bf16", "gate": 1, "grad": True},
        # wide rows in 32 bits, a gate for each sequence
        {"name": "norms_wide_f32", "kind": "norms", "rows": 4096, "d": 8192, "dtype": "f32", "gate": 512, "grad": True},
        # the gated norm of every head of the training step
        {"name": "gated_train", "kind": "gated", "rows": 16384, "heads": 16, "d": 128, "dtype": "bf16", "grad": True},
    ]


def between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "train", "train", "step", "norms", "gated"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    small = 8 if dtype == "f32" else 1
    if kind in ("prompt", "train"):
        h = rng.choice([4, 8, 12, 16, 24])
        hq, hk, hv = rng.choice([(h, h, h), (h, h, h), (h, h // 4, h // 4), (h // 4, h // 4, h)])
        most = (400000 if kind == "prompt" else 200000) // small  # tokens times heads
        t = between(rng, 2, min(32768, most // h))
        b = between(rng, 1, max(1, min(32, most // (h * t))))
        return attention_case(kind, b, t, h, hq, hk, hv, rng.choice([64, 96, 128, 128]), rng.choice([64, 80, 128, 128]), dtype,
                              rng.choice(["token", "head"]), rng.random() < 0.5, rng.random() < 0.25)
    if kind == "step":
        h = rng.choice([4, 8, 16, 24])
        b = between(rng, 1, 160)
        return {"kind": "step", "b": b, "h": h, "hq": h, "hk": rng.choice([h, h // 4]), "hv": h, "kd": rng.choice([64, 96, 128]),
                "vd": rng.choice([64, 80, 128]), "dtype": dtype, "pool": b + rng.randrange(40)}
    if kind == "norms":
        d = rng.choice([768, 1000, 1024, 2048, 4096, 5120, 8192])
        rows = between(rng, 1, (1 << 24) // d)
        gate = rng.choice([0, 1, 1, between(rng, 1, rows)])
        return {"kind": "norms", "rows": rows, "d": d, "dtype": dtype, "gate": gate, "grad": rng.random() < 0.6}
    d, heads = rng.choice([64, 80, 128, 256]), rng.choice([4, 8, 16])
    return {"kind": "gated", "rows": between(rng, 1, (1 << 24) // (d * heads)), "heads": heads, "d": d, "dtype": dtype,
            "grad": rng.random() < 0.6}


# --------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape, to=dt, spread=1.0, about=0.0):
        return torch.randn(*shape, device="cuda", generator=g).mul_(spread).add_(about).to(to)

    s = {"case": case}
    if case["kind"] in ("prompt", "train"):
        b, t, h, kd, vd = (case[n] for n in ("b", "t", "h", "kd", "vd"))
        s["q"], s["k"], s["v"] = normal(b, t, case["hq"], kd), normal(b, t, case["hk"], kd), normal(b, t, case["hv"], vd)
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
            for n in ("q", "k", "v", "log_a", "state0"):
                if s[n] is not None:
                    s[n].requires_grad_()
    elif case["kind"] == "step":
        b, h, kd, vd = (case[n] for n in ("b", "h", "kd", "vd"))
        s["q"], s["k"], s["v"] = normal(b, case["hq"], kd), normal(b, case["hk"], kd), normal(b, case["hv"], vd)
        s["log_a"] = torch.nn.functional.logsigmoid(normal(b, h, to=torch.float32, about=3.0))
        s["state"] = normal(case["pool"], h, kd, vd, to=torch.float32)
        s["slots"] = torch.randperm(case["pool"], device="cuda", generator=g)[:b].to(torch.int32)
    elif case["kind"] == "norms":
        rows, d, per = case["rows"], case["d"], case["gate"]
        s["x"], s["branch"] = normal(rows, d), normal(rows, d, spread=0.7)
        s["gate"] = None
        if per == 1:  # a gate for each row
            s["gate"] = normal(rows, d, spread=0.5, about=1.0)
        elif per > 1:  # a gate for each sequence of `per` rows
            rows = per * max(1, rows // per)
            s["x"], s["branch"] = (s[n][:rows].reshape(rows // per, per, d) for n in ("x", "branch"))
            s["gate"] = normal(rows // per, 1, d, spread=0.5, about=1.0)
        s["pre"], s["post"] = normal(d, spread=0.1, about=1.0), normal(d, spread=0.1, about=1.0)
        s["scale"] = 0.5
        if case["grad"]:
            s["dr"], s["dy"] = (normal(*s["x"].shape) for _ in range(2))
            for n in ("x", "branch", "gate", "pre", "post"):
                if s[n] is not None:
                    s[n].requires_grad_()
    else:
        rows, heads, d = case["rows"], case["heads"], case["d"]
        s["x"], s["gate"] = normal(rows, heads, d, spread=3.0), normal(rows, heads, d)
        s["weight"] = normal(d, spread=0.1, about=1.0)
        if case["grad"]:
            s["dy"] = normal(rows, heads, d)
            for n in ("x", "gate", "weight"):
                s[n].requires_grad_()
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


def plain_attention(q, k, v, log_a, state0, scale, lengths):
    b, t = q.shape[:2]
    h = log_a.shape[-1]
    dt = q.dtype
    q, k, v = (to_heads(x.float(), h) for x in (q, k, v))
    a = log_a.float().expand(b, t, h)
    if lengths is not None:
        live = (torch.arange(t, device=q.device) < lengths[:, None])[..., None]
        k, v, a = k * live[..., None], v * live[..., None], a * live
    n = -(-t // CHUNK)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, n * CHUNK - t)).unflatten(1, (n, CHUNK))  # noqa: E731
    q, k, v = (cut(x).permute(0, 3, 1, 2, 4) for x in (q, k, v))  # [b, h, n, chunk, width]
    a = cut(a).permute(0, 3, 1, 2)
    c = a.cumsum(-1)
    o = ((q @ k.transpose(-1, -2)) * sums_between(a).exp()) @ v
    new = (k * (c[..., -1:] - c).exp().unsqueeze(-1)).transpose(-1, -2) @ v  # what each chunk adds to the state
    first = torch.zeros_like(new[:, :, 0]) if state0 is None else state0.float()
    every = torch.cat([first.unsqueeze(2), new], 2).flatten(3)
    carry = sums_between(torch.cat([torch.zeros_like(c[:, :, :1, -1]), c[..., -1]], -1)).exp()
    states = (carry @ every).unflatten(3, new.shape[3:])  # before each chunk, and at the end
    o = o + (q @ states[:, :, :-1]) * c.exp().unsqueeze(-1)
    o = (o * scale).permute(0, 2, 3, 1, 4).flatten(1, 2)[:, :t]
    if lengths is not None:
        o = o * live[..., None]
    return o.to(dt), states[:, :, -1]


def plain_step(q, k, v, log_a, state, scale, slots):
    h = log_a.shape[-1]
    at = slots.long()
    k, v, qf = (to_heads(x.float(), h) for x in (k, v, q))
    new = state[at] * log_a.float().exp()[..., None, None] + k.unsqueeze(-1) * v.unsqueeze(-2)
    state[at] = new
    return ((qf * scale).unsqueeze(-2) @ new).squeeze(-2).to(q.dtype)


def plain_rms(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def plain_norms(x, branch, pre, post, gate, scale):
    n = plain_rms(branch.float()) * post.float()
    r = x.float() + scale * (n if gate is None else gate.float() * n)
    return r.to(x.dtype), (plain_rms(r) * pre.float()).to(x.dtype)


def plain_gated(x, gate, weight):
    z = gate.float()
    return (plain_rms(x.float()) * weight.float() * (z / (1 + (-z).exp()))).to(x.dtype)


# ------------------------------------------------------------------------------------------- the pass

def gradients(outputs, grads, inputs):
    names = [n for n, x in inputs.items() if x is not None]
    pairs = [(o, g) for o, g in zip(outputs, grads) if g is not None]
    got = torch.autograd.grad([o for o, _ in pairs], [inputs[n] for n in names], [g for _, g in pairs])
    return {"d" + n: g for n, g in zip(names, got)}


def run(s):
    case = s["case"]
    if own:
        from paper_2311_06281_b200 import heinsen_attention as ha
    if case["kind"] in ("prompt", "train"):
        scale = case["kd"] ** -0.5
        if own:
            o, state = ha.decay_attention(s["q"], s["k"], s["v"], s["log_a"], s["state0"], scale=scale, lengths=s["lengths"])
        else:
            o, state = plain_attention(s["q"], s["k"], s["v"], s["log_a"], s["state0"], scale, s["lengths"])
        out = {"o": o, "state": state}
        if case["kind"] == "train":
            out.update(gradients([o, state], [s["do"], s["dstate"]], {n: s[n] for n in ("q", "k", "v", "log_a", "state0")}))
        return out
    if case["kind"] == "step":
        call = ha.decay_attention_step if own else plain_step
        o = call(s["q"], s["k"], s["v"], s["log_a"], s["state"], scale=case["kd"] ** -0.5, slots=s["slots"])
        return {"o": o, "state": s["state"]}
    if case["kind"] == "norms":
        if own:
            r, y = ha.block_norms(s["x"], s["branch"], s["pre"], post_weight=s["post"], gate=s["gate"], scale=s["scale"], eps=EPS)
        else:
            r, y = plain_norms(s["x"], s["branch"], s["pre"], s["post"], s["gate"], s["scale"])
        out = {"r": r, "y": y}
        if case["grad"]:
            out.update(gradients([r, y], [s["dr"], s["dy"]], {n: s[n] for n in ("x", "branch", "gate", "pre", "post")}))
        return out
    y = ha.gated_norm(s["x"], s["gate"], s["weight"], eps=EPS) if own else plain_gated(s["x"], s["gate"], s["weight"])
    out = {"y": y}
    if case["grad"]:
        out.update(gradients([y], [s["dy"]], {n: s[n] for n in ("x", "gate", "weight")}))
    return out


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] in ("prompt", "train"):
        b, t, h, hq, hk, hv, kd, vd = (case[n] for n in ("b", "t", "h", "hq", "hk", "hv", "kd", "vd"))
        qkv = b * t * (hq * kd + hk * kd + hv * vd) * size
        decays = b * t * h * 4 if case["decay"] == "token" else h * 4
        state = b * h * kd * vd * 4
        flops = 4 * b * t * h * kd * vd  # the update and the readout of the recurrent form
        moved = qkv + decays + b * t * h * vd * size + state * (2 if case["state"] else 1)
        if case["kind"] == "train":  # dO in, gradients out
            moved += qkv + decays + b * t * h * vd * size + (2 * state if case["state"] else 0)
            flops *= 3.5
        return {"bytes": moved, "flops": flops}
    if case["kind"] == "step":
        b, h, kd, vd = (case[n] for n in ("b", "h", "kd", "vd"))
        state = b * h * kd * vd
        rows = b * (case["hq"] * kd + case["hk"] * kd + case["hv"] * vd + h * vd) * size
        return {"bytes": 8 * state + rows + 4 * b * (h + 1), "flops": 5 * state}
    if case["kind"] == "norms":
        per = case["gate"]
        rows = case["rows"] if per <= 1 else per * max(1, case["rows"] // per)
        n = rows * case["d"]
        gate = 0 if per == 0 else n // per
        moved = (4 * n + gate + 2 * case["d"]) * size
        if case["grad"]:  # dr, dy in; dx, dbranch, dgate and the weights' gradients out
            moved += (4 * n + gate + 2 * case["d"]) * size
        return {"bytes": moved, "flops": n * (30 if case["grad"] else 10)}
    n = case["rows"] * case["heads"] * case["d"]
    return {"bytes": (6 if case["grad"] else 3) * n * size, "flops": n * (30 if case["grad"] else 10)}


# ------------------------------------------------------------------------------- from the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    d = {n: x.detach().double() if isinstance(x, torch.Tensor) and x.is_floating_point() else x for n, x in s.items()}
    with torch.no_grad():
        return {"prompt": exact_attention, "train": exact_attention, "step": exact_step, "norms": exact_norms,
                "gated": exact_gated}[case["kind"]](case, d)


def exact_attention(case, d):
    """Every pair of tokens by itself: W_ij = scale exp(sum of the decays after j up to i), rows in blocks."""
    b, t, h, kd, vd = (case[n] for n in ("b", "t", "h", "kd", "vd"))
    scale, train, dev = kd ** -0.5, case["kind"] == "train", "cuda"
    f8 = dict(dtype=torch.float64, device=dev)
    out = {"o": torch.zeros(b, t, h, vd, **f8), "state": torch.zeros(b, h, kd, vd, **f8)}
    if train:
        out.update({"d" + n: torch.zeros_like(d[n]) for n in ("q", "k", "v", "log_a", "state0") if d[n] is not None})
    for i in range(b):
        n = t if d["lengths"] is None else int(d["lengths"][i])
        for j in range(h):
            jq, jk, jv = (j * case[x] // h for x in ("hq", "hk", "hv"))
            q, k, v = d["q"][i, :n, jq], d["k"][i, :n, jk], d["v"][i, :n, jv]
            a = d["log_a"][i, :n, j] if case["decay"] == "token" else d["log_a"][j].expand(n)
            c = a.cumsum(0)
            s0 = d["state0"][i, j] if d["state0"] is not None else torch.zeros(kd, vd, **f8)
            end = c[-1] if n else torch.zeros((), **f8)
            late = (end - c).exp()[:, None]
            last = s0 * end.exp() + (k * late).T @ v
            out["state"][i, j] = last
            if train:
                do = d["do"][i, :n, j]
                ds = d["dstate"][i, j] if d["dstate"] is not None else torch.zeros(kd, vd, **f8)
                dq, dk, dv = (torch.zeros_like(x) for x in (q, k, v))
                through = torch.zeros(n, **f8)  # what the loss owes to every exponent, to be summed from the end
            for lo in range(0, n, 4096):
                hi = min(n, lo + 4096)
                rows = torch.arange(lo, hi, device=dev)
                gap = c[lo:hi, None] - c[None, :hi]
                w = torch.where(rows[:, None] >= torch.arange(hi, device=dev), gap, -math.inf).exp() * scale
                early = c[lo:hi, None].exp() * scale
                p = w * (q[lo:hi] @ k[:hi].T)
                out["o"][i, lo:hi, j] = p @ v[:hi] + early * (q[lo:hi] @ s0)
                if train:
                    e = do[lo:hi] @ v[:hi].T
                    back = early * (do[lo:hi] @ s0.T)
                    dq[lo:hi] += (w * e) @ k[:hi] + back
                    dk[:hi] += (w * e).T @ q[lo:hi]
                    dv[:hi] += p.T @ do[lo:hi]
                    through[lo:hi] += (p * e).sum(1) + (q[lo:hi] * back).sum(1)
                    through[:hi] -= (p * e).sum(0)
                    if "dstate0" in out:
                        out["dstate0"][i, j] += (q[lo:hi] * early).T @ do[lo:hi]
            if train and n:
                far = late * (v @ ds.T)
                through -= (k * far).sum(1)
                through[-1] += (last * ds).sum()
                da = through.flip(0).cumsum(0).flip(0)
                out["dq"][i, :n, jq] += dq
                out["dk"][i, :n, jk] += dk + far
                out["dv"][i, :n, jv] += dv + late * (k @ ds)
                if case["decay"] == "token":
                    out["dlog_a"][i, :n, j] += da
                else:
                    out["dlog_a"][j] += da.sum()
            if train and "dstate0" in out:
                out["dstate0"][i, j] += ds * end.exp()
    return out


def exact_step(case, d):
    b, h = case["b"], case["h"]
    at = d["slots"].long()
    head = torch.arange(h, device="cuda")
    q, k, v = (d[n][:, head * case["h" + n] // h] for n in ("q", "k", "v"))
    state = d["state"].clone()
    state[at] = torch.einsum("bh,bhkv->bhkv", d["log_a"].exp(), state[at]) + torch.einsum("bhk,bhv->bhkv", k, v)
    return {"o": torch.einsum("bhk,bhkv->bhv", q, state[at]) * case["kd"] ** -0.5, "state": state}


def back_through_rms(x, dn):
    """The gradient of x / sqrt(mean x^2 + eps), given that of its result."""
    root = (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    n = x / root
    return (dn - n * (n * dn).mean(-1, keepdim=True)) / root, n


def exact_norms(case, d):
    x, h, pre, post, scale = (d[n] for n in ("x", "branch", "pre", "post", "scale"))
    gate = torch.ones((), dtype=torch.float64, device="cuda") if d["gate"] is None else d["gate"]
    n = h / (h.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    r = x + scale * gate * n * post
    out = {"r": r, "y": r / (r.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * pre}
    if case["grad"]:
        dr, m = back_through_rms(r, d["dy"] * pre)
        dr = dr + d["dr"]
        per_gate = dr * scale * n * post
        dh, n = back_through_rms(h, dr * scale * gate * post)
        flat = lambda z: z.reshape(-1, z.shape[-1]).sum(0)  # noqa: E731
        out.update({"dx": dr, "dbranch": dh, "dpre": flat(d["dy"] * m), "dpost": flat(dr * scale * gate * n)})
        if d["gate"] is not None:
            out["dgate"] = per_gate if case["gate"] == 1 else per_gate.sum(1, keepdim=True)
    return out


def exact_gated(case, d):
    x, z, w = d["x"], d["gate"], d["weight"]
    open_ = torch.sigmoid(z)
    n = x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
    out = {"y": n * w * z * open_}
    if case["grad"]:
        dx, n = back_through_rms(x, d["dy"] * w * z * open_)
        out.update({"dx": dx, "dgate": d["dy"] * n * w * open_ * (1 + z * (1 - open_)),
                    "dweight": (d["dy"] * n * z * open_).sum((0, 1))})
    return out
