"""Timed workloads of the gated delta rule and of the channels-last group norm: what a program around a ViG block has them do.

A case names what is done ("do") and its sizes:

  mix     the gated delta rule over whole sequences: B images, H heads, L tokens, head sizes dk and dv, either direction, with an
          initial and a final state ("states") where a sequence is continued
  train   the same with its gradient: one training step of the mixer
  step    one new token of B sequences against their states, which are updated in place
  norm    group norm with an activation over [B, Hh, Ww, C] images
  tnorm   the same with its gradient

Values: q and k of unit length, v and d_out ~ N(0, 1), log alpha = logsigmoid(g) / 16 with g ~ N(gate_mean, 1) as everywhere in this
library, beta = sigmoid of N(0, 1), states ~ N(0, 0.3^2); images ~ N(0.2, 1) with weights around one.

`own` False: the operators in elementary torch operations, fp32 inside and rounded once at the end; the delta rule by chunks of 64
tokens (a triangular system per chunk, states carried from chunk to chunk), gradients by reverse mode through that.
"""
import math

import torch

own = False

TAU = 16.0
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "silu", "gelu")
EPS = 1e-5


def _seq(name, do, B, H, L, dk, dv, dtype="bf16", gate_mean=0.0, reverse=False, states=False):
    return {"name": name, "do": do, "B": B, "H": H, "L": L, "dk": dk, "dv": dv, "dtype": dtype, "gate_mean": gate_mean, "reverse": reverse, "states": states}


def _img(name, do, B, Hh, Ww, C, groups, dtype="bf16", act="silu"):
    return {"name": name, "do": do, "B": B, "Hh": Hh, "Ww": Ww, "C": C, "groups": groups, "dtype": dtype, "act": act}


def listed():
    return [
        # ordinary evaluation batch at 224 x 224, the larger heads with slow gates
        _seq("mix_b224", "mix", 64, 12, 196, 32, 64, gate_mean=2.0),
        # a high-resolution batch, few long sequences, the direction from the last patch to the first
        _seq("mix_t1024_reverse", "mix", 8, 4, 4096, 24, 48, reverse=True),
        # a long prefix that later single steps continue: heads of 128, initial and final state
        _seq("mix_prefix_4096", "mix", 2, 16, 4096, 128, 128, gate_mean=2.0, states=True),
        # training: ViG-B at 224, ViG-T at 1024
        _seq("train_b224", "train", 64, 12, 196, 32, 64, gate_mean=2.0),
        _seq("train_t1024", "train", 8, 4, 4096, 24, 48),
        # full-precision training of a small batch (validating a run, debugging a loss), continued from a state
        _seq("train_s224_f32", "train", 8, 6, 196, 32, 64, dtype="f32", states=True),
        # one token of one sequence: latency
        _seq("step_one", "step", 1, 4, 1, 24, 48),
        # one token of many sequences: the states' way through memory
        _seq("step_256", "step", 256, 16, 1, 128, 128, gate_mean=2.0),
        # norm behind the depth-wise convolution of one 1024 x 1024 image
        _img("norm_1024_one_image", "norm", 1, 64, 64, 192, 8),
        # the convolutional stem's resolution, an evaluation batch
        _img("norm_stem", "norm", 64, 56, 56, 96, 32),
        # training: a block of ViG-B at 224, groups of three channels of the stem at full precision
        _img("tnorm_b224", "tnorm", 64, 14, 14, 768, 32),
        _img("tnorm_stem_f32", "tnorm", 16, 56, 56, 96, 32, dtype="f32", act="gelu"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any of the things done, from a single token or a small image up to the listed batches."""
    do = rng.choice(("mix", "mix", "train", "train", "step", "norm", "tnorm"))
    if do in ("norm", "tnorm"):
        dtype = rng.choice(("bf16", "bf16", "f32"))
        per = rng.choice((1, 2, 3, 4, 8, 12, 16, 24, 32, 64))
        groups = rng.choice([g for g in (1, 2, 4, 6, 8, 16, 24, 32) if (g * per) % 8 == 0 and 16 <= g * per <= 1536])
        C = groups * per
        most = (9_000_000 if do == "norm" else 5_000_000) // C
        Hh, Ww = _log_uniform(rng, 1, 112), _log_uniform(rng, 1, 112)
        if Hh * Ww * per < 32:   # (the gradient of a statistic over a handful of values is all cancellation)
            Hh = -(-32 // (Ww * per))
        B = _log_uniform(rng, 1, max(1, min(256, most // (Hh * Ww))))
        return {k: v for k, v in _img("", do, B, Hh, Ww, C, groups, dtype, rng.choice(ACTS)).items() if k != "name"}
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    size = (lambda hi: 8 * rng.randint(2, hi // 8)) if rng.random() < 0.75 else (lambda hi: rng.randint(5, hi))
    dk, dv = size(128), size(128)
    gate_mean = rng.choice((-1.0, 0.0, 2.0, 4.0))
    if do == "step":
        BH = _log_uniform(rng, 1, max(1, min(8192, 60_000_000 // (dk * dv))))
        L = 1
    else:
        L = _log_uniform(rng, 1, 8192 if do == "mix" else 4096)
        most = 2_000_000_000 if do == "mix" else 300_000_000
        wide = 30_000_000 if do == "mix" else 14_000_000
        if dtype == "f32":
            most, wide = most // 8, wide // 4
        BH = _log_uniform(rng, 1, max(1, min(4096, most // (L * dk * dv), wide // (L * (dk + dv)))))
    H = rng.choice([h for h in (1, 2, 3, 4, 6, 12, 16, 24) if h <= BH])
    c = _seq("", do, max(1, BH // H), H, L, dk, dv, dtype, gate_mean, rng.random() < 0.4 and do != "step", rng.random() < 0.5 and do != "step")
    return {k: v for k, v in c.items() if k != "name"}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = TYPES[case["dtype"]]

    def normal(*shape, mean=0.0, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std + mean

    if case["do"] in ("norm", "tnorm"):
        B, Hh, Ww, C, G = (case[n] for n in ("B", "Hh", "Ww", "C", "groups"))
        s = {"case": case, "x": normal(B, Hh, Ww, C, mean=0.2).to(T), "weight": normal(C, mean=1.0, std=0.2).to(T), "bias": normal(C, std=0.2).to(T)}
        s["out"] = torch.empty_like(s["x"])
        if case["do"] == "tnorm":
            s["d_out"] = normal(B, Hh, Ww, C).to(T)
            s["mean"], s["rstd"] = (torch.empty(B, G, device="cuda") for _ in range(2))
            s["dx"], s["dweight"], s["dbias"] = torch.empty_like(s["x"]), torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
        return s
    B, H, L, dk, dv = (case[n] for n in ("B", "H", "L", "dk", "dv"))
    unit = lambda x: (x / x.square().sum(-1, keepdim=True).sqrt()).to(T)  # noqa: E731
    s = {"case": case, "q": unit(normal(B, H, L, dk)), "k": unit(normal(B, H, L, dk)), "v": normal(B, H, L, dv).to(T)}
    s["log_alpha"] = (torch.nn.functional.logsigmoid(normal(B, H, L, mean=case["gate_mean"])) / TAU).to(T)
    s["beta"] = torch.sigmoid(normal(B, H, L)).to(T)
    s["out"] = torch.empty_like(s["v"])
    if case["do"] == "step":
        for n in ("q", "k", "v", "out"):
            s[n] = s[n].reshape(B, H, -1)
        for n in ("log_alpha", "beta"):
            s[n] = s[n].reshape(B, H)
    if case["do"] == "step" or case["states"]:
        s["state"] = normal(B, H, dk, dv, std=0.3)
    if case["states"]:
        s["state_out"] = torch.empty_like(s["state"])
    if case["do"] == "train":
        s["d_out"] = normal(B, H, L, dv).to(T)
        for n in ("q", "k", "v", "log_alpha", "beta"):
            s["d" + n] = torch.empty_like(s[n])
        if case["states"]:
            s["d_state_out"], s["d_state"] = normal(B, H, dk, dv), torch.empty_like(s["state"])
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _plain_chunks(q, k, v, la, beta, state, C=64):
    """The gated delta rule in fp32 by chunks of C tokens: out and the last state."""
    B, H, L, dk = q.shape
    n = -(-L // C)
    cut = lambda x: torch.nn.functional.pad(x, (0, 0, 0, n * C - L)).reshape(B, H, n, C, -1)  # noqa: E731
    q, k, v, la, beta = cut(q), cut(k), cut(v), cut(la[..., None]), cut(beta[..., None])
    b = la.cumsum(-2)
    low = torch.ones(C, C, dtype=torch.bool, device=q.device).tril()
    decay = torch.exp((b - b.transpose(-1, -2)).masked_fill(~low, 0.0)) * low
    system = torch.eye(C, device=q.device) + (beta * (k @ k.transpose(-1, -2)) * decay).tril(-1)
    both = torch.linalg.solve_triangular(system, torch.cat((beta * v, beta * b.exp() * k), -1), upper=False, unitriangular=True)
    u0, w = both.split((v.shape[-1], dk), -1)
    scores = (q @ k.transpose(-1, -2)) * decay
    qb, kb, last = q * b.exp(), k * (b[..., -1:, :] - b).exp(), b[..., -1:, :].exp()
    S = q.new_zeros(B, H, dk, v.shape[-1]) if state is None else state
    out = []
    for i in range(n):
        u = u0[:, :, i] - w[:, :, i] @ S
        out.append(qb[:, :, i] @ S + scores[:, :, i] @ u)
        S = last[:, :, i] * S + kb[:, :, i].transpose(-1, -2) @ u
    return torch.stack(out, 2).reshape(B, H, n * C, -1)[:, :, :L], S


def _plain_mix(s, grads):
    case = s["case"]
    flip = (lambda x: x.flip(2)) if case["reverse"] else (lambda x: x)
    names = ["q", "k", "v", "log_alpha", "beta"]
    x = [s[n].float().requires_grad_(grads) for n in names]
    state = s["state"].clone().requires_grad_(grads) if case["states"] else None
    with torch.set_grad_enabled(grads):
        out, last = _plain_chunks(*(flip(t) for t in x), state)
        out = flip(out)
    made = {"out": out.detach().to(s["v"].dtype)}
    if case["states"]:
        made["state_out"] = last.detach()
    if grads:
        ends, ups = ([out, last], [s["d_out"].float(), s["d_state_out"]]) if case["states"] else ([out], [s["d_out"].float()])
        got = torch.autograd.grad(ends, x + ([state] if case["states"] else []), ups)
        made.update({"d" + n: t.to(s[n].dtype) for n, t in zip(names, got)})
        if case["states"]:
            made["d_state"] = got[5]
    return made


def _plain_step(s):
    q, k, v, beta = (s[n].float() for n in ("q", "k", "v", "beta"))
    S = s["state"] * s["log_alpha"].float().exp()[..., None, None]
    u = beta[..., None] * (v - (k[..., None] * S).sum(-2))
    S = S + k[..., None] * u[..., None, :]
    s["state"].copy_(S)
    return {"out": (q[..., None] * S).sum(-2).to(s["v"].dtype), "state": s["state"]}


def _activation(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z * 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) if act == "gelu" else z


def _plain_norm(s, grads):
    case = s["case"]
    B, Hh, Ww, C, G = (case[n] for n in ("B", "Hh", "Ww", "C", "groups"))
    x, w, b = (s[n].float().requires_grad_(grads) for n in ("x", "weight", "bias"))
    with torch.set_grad_enabled(grads):
        y = x.reshape(B, Hh * Ww, G, C // G)
        y = y - y.mean((1, 3), keepdim=True)
        y = y / (y.square().mean((1, 3), keepdim=True) + EPS).sqrt()
        out = _activation(y.reshape(B, Hh, Ww, C) * w + b, case["act"])
    made = {"out": out.detach().to(s["x"].dtype)}
    if grads:
        got = torch.autograd.grad(out, (x, w, b), s["d_out"].float())
        made.update({"d" + n: t.to(s["x"].dtype) for n, t in zip(("x", "weight", "bias"), got)})
    return made


def run(s):
    case = s["case"]
    do = case["do"]
    if not own:
        if do in ("norm", "tnorm"):
            return _plain_norm(s, do == "tnorm")
        return _plain_step(s) if do == "step" else _plain_mix(s, do == "train")
    import paper_2405_18425_b200 as vig

    if do in ("norm", "tnorm"):
        G, act = case["groups"], case["act"]
        if do == "norm":
            vig.vig_group_norm(s["x"], s["weight"], s["bias"], s["out"], G, EPS, act)
            return {"out": s["out"]}
        vig.vig_group_norm(s["x"], s["weight"], s["bias"], s["out"], G, EPS, act, mean=s["mean"], rstd=s["rstd"])
        vig.vig_group_norm_bwd(s["x"], s["weight"], s["bias"], s["mean"], s["rstd"], s["d_out"], s["dx"], s["dweight"], s["dbias"], G, act)
        return {n: s[n] for n in ("out", "dx", "dweight", "dbias")}
    x = [s[n] for n in ("q", "k", "v", "log_alpha", "beta")]
    if do == "step":
        vig.vig_gdr_step(*x, s["state"], s["out"])
        return {"out": s["out"], "state": s["state"]}
    vig.vig_gdr_fwd(*x, s["out"], state_in=s.get("state"), state_out=s.get("state_out"), reverse=case["reverse"])
    names = ["out"] + (["state_out"] if case["states"] else [])
    if do == "train":
        grads = [s["d" + n] for n in ("q", "k", "v", "log_alpha", "beta")]
        vig.vig_gdr_bwd(*x, s["d_out"], *grads, state_in=s.get("state"), d_state_out=s.get("d_state_out"), d_state_in=s.get("d_state"), reverse=case["reverse"])
        names += ["dq", "dk", "dv", "dlog_alpha", "dbeta"] + (["d_state"] if case["states"] else [])
    return {n: s[n] for n in names}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------
def _exact_mix(s, grads):
    """Token by token; the gradient from the states of all tokens, kept."""
    case = s["case"]
    B, H, L, dk, dv = (case[n] for n in ("B", "H", "L", "dk", "dv"))
    q, k, v, la, beta = (s[n].double().reshape(B * H, L, -1) for n in ("q", "k", "v", "log_alpha", "beta"))
    alpha = la.exp()
    S = s["state"].double().reshape(B * H, dk, dv).clone() if case["states"] else torch.zeros(B * H, dk, dv, dtype=torch.float64, device="cuda")
    order = range(L - 1, -1, -1) if case["reverse"] else range(L)
    out, w, kept = torch.empty_like(v), torch.empty_like(v), {}
    for t in order:
        S = S * alpha[:, t, :, None]
        w[:, t] = v[:, t] - torch.einsum("nij,ni->nj", S, k[:, t])
        if grads:
            kept[t] = S
        S = S + k[:, t, :, None] * (beta[:, t] * w[:, t])[:, None]
        out[:, t] = torch.einsum("nij,ni->nj", S, q[:, t])
    whole = lambda x, n: x.reshape(s[n].shape)  # noqa: E731
    made = {"out": whole(out, "v")}
    if case["states"]:
        made["state_out"] = S.reshape(B, H, dk, dv)
    if grads:
        d = {n: torch.empty_like(t) for n, t in (("q", q), ("k", k), ("v", v), ("log_alpha", la), ("beta", beta))}
        do = s["d_out"].double().reshape(B * H, L, dv)
        dS = s["d_state_out"].double().reshape(B * H, dk, dv).clone() if case["states"] else torch.zeros_like(S)
        for t in reversed(order):
            low = kept.pop(t)
            u = beta[:, t] * w[:, t]
            dS = dS + q[:, t, :, None] * do[:, t, None]
            d["q"][:, t] = torch.einsum("nij,nj->ni", low + k[:, t, :, None] * u[:, None], do[:, t])
            du = torch.einsum("nij,ni->nj", dS, k[:, t])
            dw = beta[:, t] * du
            d["v"][:, t] = dw
            d["beta"][:, t] = (du * w[:, t]).sum(-1, keepdim=True)
            d["k"][:, t] = torch.einsum("nij,nj->ni", dS, u) - torch.einsum("nij,nj->ni", low, dw)
            dS = dS - k[:, t, :, None] * dw[:, None]
            d["log_alpha"][:, t] = (dS * low).sum((1, 2))[:, None]
            dS = dS * alpha[:, t, :, None]
        made.update({"d" + n: whole(x, n) for n, x in d.items()})
        if case["states"]:
            made["d_state"] = dS.reshape(B, H, dk, dv)
    return made


def _exact_norm(s, grads):
    """The gradient by its closed form."""
    case = s["case"]
    B, Hh, Ww, C, G = (case[n] for n in ("B", "Hh", "Ww", "C", "groups"))
    x, w, b = s["x"].double().reshape(B, Hh * Ww, G, C // G), s["weight"].double().reshape(G, -1), s["bias"].double().reshape(G, -1)
    var, mu = torch.var_mean(x, (1, 3), correction=0, keepdim=True)
    rstd = (var + EPS).rsqrt()
    xhat = (x - mu) * rstd
    z = xhat * w + b
    sig, phi = torch.sigmoid(z), torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    cdf = 0.5 * torch.special.erfc(-z * math.sqrt(0.5))
    y, slope = {"none": (z, torch.ones_like(z)), "silu": (z * sig, sig * (1 + z * (1 - sig))), "gelu": (z * cdf, cdf + z * phi)}[case["act"]]
    made = {"out": y.reshape(B, Hh, Ww, C)}
    if grads:
        g = s["d_out"].double().reshape(x.shape) * slope
        gw = g * w
        dx = rstd * (gw - gw.mean((1, 3), keepdim=True) - xhat * (gw * xhat).mean((1, 3), keepdim=True))
        made.update(dx=dx.reshape(B, Hh, Ww, C), dweight=(g * xhat).sum((0, 1)).reshape(C), dbias=g.sum((0, 1)).reshape(C))
    return made


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] in ("norm", "tnorm"):
        return _exact_norm(s, case["do"] == "tnorm")
    if case["do"] == "step":
        q, k, v, la, beta, S = (s[n].double() for n in ("q", "k", "v", "log_alpha", "beta", "state"))
        S = torch.einsum("bh,bhij->bhij", la.exp(), S)
        u = beta[..., None] * (v - torch.einsum("bhij,bhi->bhj", S, k))
        S = S + torch.einsum("bhi,bhj->bhij", k, u)
        return {"out": torch.einsum("bhij,bhi->bhj", S, q), "state": S}
    return _exact_mix(s, case["do"] == "train")


def work(case):
    """Each input read once, each output written once; the recurrence's multiplications and additions (decay, retrieval, update and
    read-out of a dk x dv state per token; with the gradient the walk of its adjoint and the four products with both states)."""
    e = 2 if case["dtype"] == "bf16" else 4
    if case["do"] in ("norm", "tnorm"):
        n = case["B"] * case["Hh"] * case["Ww"] * case["C"]
        c = case["C"]
        return {"bytes": (4 * n + 4 * c) * e, "flops": 40 * n} if case["do"] == "tnorm" else {"bytes": (2 * n + 2 * c) * e, "flops": 15 * n}
    BH, L, dk, dv = case["B"] * case["H"], case["L"], case["dk"], case["dv"]
    state = 4 * BH * dk * dv
    if case["do"] == "step":
        return {"bytes": BH * (2 * dk + 2 * dv + 2) * e + 2 * state, "flops": 7 * BH * dk * dv}
    if case["do"] == "mix":
        return {"bytes": BH * L * (2 * dk + 2 * dv + 2) * e + (2 * state if case["states"] else 0), "flops": 7 * BH * L * dk * dv}
    return {"bytes": BH * L * (4 * dk + 4 * dv + 4) * e + (4 * state if case["states"] else 0), "flops": 23 * BH * L * dk * dv}
