"""Timed workloads of the selective state space scan, its causal convolution and the RMS norm with a residual: what a program around a
block with that mixer has them do.

A case names what is done ("do") and its sizes:

  scan    the selective scan over whole sequences: B images, L tokens, C channels in G groups that share their rows of Bt and Ct, N
          states a channel, either direction, gated by z, with an initial and a final state ("states") where a sequence is continued
  train   the same with its gradient: one training step of the mixer
  step    one new token of B sequences against their states, which are updated in place
  conv    the causal convolution of width K with SiLU in front of the scan
  tconv   the same with its gradient
  cstep   its single-token form, the window of past tokens updated in place
  norm    RMS norm of B L rows of C values, the residual added before it and handed on
  norm8   the same with its result in 8 bits: a scale for every row (block 0) or for every 128 values (block 128)
  tnorm   the norm and its gradient

Values: as behind a projection.  x, z, Bt and Ct ~ N(0, 1), z beside x and Ct beside Bt in the rows that one projection writes; A = -(1 .. N)
up to a factor around one; step sizes softplus(dt + bias) with dt ~ N(0, 0.5^2) and biases that put softplus(bias) log-uniformly into
[0.001, 0.1]; states and gradients ~ N(0, 1); the residual ~ N(0, 2^2).

`own` False: the operators in elementary torch operations, fp32 inside and rounded once at the end; the recurrence by doubling (log2 L
passes over all states at once), gradients by the adjoint recurrence, written out.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def _seq(name, do, B, L, C, N, G=1, dtype="bf16", reverse=False, states=False):
    return {"name": name, "do": do, "B": B, "L": L, "C": C, "N": N, "G": G, "dtype": dtype, "reverse": reverse, "states": states}


def _conv(name, do, B, L, C, K=4, dtype="bf16", reverse=False, states=False):
    return {"name": name, "do": do, "B": B, "L": L, "C": C, "K": K, "dtype": dtype, "reverse": reverse, "states": states}


def _rows(name, do, B, L, C, dtype="bf16", block=0, residual=True):
    return {"name": name, "do": do, "B": B, "L": L, "C": C, "dtype": dtype, "block": block, "residual": residual}


def listed():
    return [
        # ordinary evaluation batch at 224 x 224, width 768 expanded by a half
        _seq("scan_b224", "scan", 64, 196, 1152, 16),
        # a high-resolution batch, few long sequences, the direction from the last patch to the first
        _seq("scan_t1024_reverse", "scan", 8, 4096, 384, 16, reverse=True),
        # one long prefix that later single steps continue: initial and final state
        _seq("scan_prefix_16384", "scan", 1, 16384, 768, 16, states=True),
        # training: ViG-B's width at 224
        _seq("train_b224", "train", 64, 196, 1152, 16),
        # full-precision training of a small batch (validating a run), two groups, continued from a state
        _seq("train_s224_f32", "train", 8, 196, 768, 8, G=2, dtype="f32", states=True),
        # one token of one sequence: latency
        _seq("step_one", "step", 1, 1, 384, 16),
        # one token of many sequences: the states' way through memory
        _seq("step_256", "step", 256, 1, 1152, 16),
        # the convolution in front of the high-resolution scan, and a training step of it at 224
        _conv("conv_t1024_reverse", "conv", 8, 4096, 384, reverse=True),
        _conv("tconv_b224", "tconv", 64, 196, 1152),
        # the norm of one image's tokens, its result in 8 bits by blocks: latency
        _rows("norm8_one_image", "norm8", 1, 196, 768, block=128),
        # the norm of a batch, its result in 8 bits by rows for a projection in 8 bits
        _rows("norm8_b224", "norm8", 64, 196, 768),
        # training, the high-resolution batch at full precision
        _rows("tnorm_t1024_f32", "tnorm", 8, 4096, 192, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any of the things done, from a single token up to the listed batches."""
    do = rng.choice(("scan", "scan", "train", "train", "step", "conv", "tconv", "cstep", "norm", "norm8", "tnorm"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if do in ("norm", "norm8", "tnorm"):
        C = 8 * _log_uniform(rng, 1, 512)
        L = _log_uniform(rng, 1, 4096)
        B = _log_uniform(rng, 1, max(1, min(256, 9_000_000 // (L * C))))
        c = _rows("", do, B, L, C, dtype, rng.choice((0, 128)) if do == "norm8" else 0, rng.random() < 0.7)
        return {k: v for k, v in c.items() if k != "name"}
    G = rng.choice((1, 1, 1, 2)) if do in ("scan", "train", "step") else 1
    C = 8 * G * _log_uniform(rng, 1, 192 // G)
    if do in ("conv", "tconv", "cstep"):
        L = 1 if do == "cstep" else _log_uniform(rng, 1, 8192)
        B = _log_uniform(rng, 1, max(1, min(256, 12_000_000 // (L * C))))
        c = _conv("", do, B, L, C, rng.choice((2, 3, 4, 4)), dtype, rng.random() < 0.4 and do != "cstep", rng.random() < 0.5 and do != "cstep")
        return {k: v for k, v in c.items() if k != "name"}
    N = rng.choice((16, 16, 16, 8, 4, 1, rng.randint(2, 32)))
    L = 1 if do == "step" else _log_uniform(rng, 1, 12288 if do == "scan" else 4096)
    most = 6_000_000 if do == "step" else 200_000_000 // (L * 2 ** (do == "train"))
    B = _log_uniform(rng, 1, max(1, min(256, most // (C * N))))
    c = _seq("", do, B, L, C, N, G, dtype, rng.random() < 0.4 and do != "step", rng.random() < 0.5 and do != "step")
    return {k: v for k, v in c.items() if k != "name"}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = TYPES[case["dtype"]]
    B, L, C, do = (case[n] for n in ("B", "L", "C", "do"))

    def normal(*shape, mean=0.0, std=1.0):
        return torch.randn(shape, generator=g, device="cuda") * std + mean

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo

    s = {"case": case}
    if do in ("norm", "norm8", "tnorm"):
        s["x"], s["weight"] = normal(B, L, C).to(T), normal(C, mean=1.0, std=0.2).to(T)
        if case["residual"]:
            s["residual"], s["sum"] = normal(B, L, C, std=2.0).to(T), torch.empty(B, L, C, device="cuda", dtype=T)
        if do == "norm8":
            s["out"] = torch.empty(B, L, C, device="cuda", dtype=torch.float8_e4m3fn)
            s["scales"] = torch.empty(B, L, -(-C // 128) if case["block"] else 1, device="cuda")
        else:
            s["out"] = torch.empty_like(s["x"])
        if do == "tnorm":
            s["d_out"], s["rstd"] = normal(B, L, C).to(T), torch.empty(B, L, device="cuda")
            s["dx"], s["dweight"] = torch.empty_like(s["x"]), torch.empty_like(s["weight"])
            if case["residual"]:
                s["d_sum"] = normal(B, L, C).to(T)   # what comes back along the residual stream
        return s
    if do in ("conv", "tconv", "cstep"):
        K = case["K"]
        xz = normal(B, L, 2 * C).to(T)   # one projection writes x and the gate side by side
        s["x"], s["out"] = xz[..., :C], torch.empty(B, L, C, device="cuda", dtype=T)
        s["weight"], s["bias"] = normal(C, K, std=K ** -0.5).to(T), normal(C, std=0.2).to(T)
        if do == "cstep" or case["states"]:
            s["state"] = normal(B, K - 1, C).to(T)
        if do == "cstep":
            s["x"], s["out"] = s["x"][:, 0], s["out"][:, 0]
        if case["states"]:
            s["state_out"] = torch.empty_like(s["state"])
        if do == "tconv":
            s["d_out"], s["dxz"] = normal(B, L, C).to(T), torch.zeros(B, L, 2 * C, device="cuda", dtype=T)
            s["dx"], s["dweight"], s["dbias"] = s["dxz"][..., :C], torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
            if case["states"]:
                s["d_state_out"], s["d_state"] = normal(B, K - 1, C).to(T), torch.empty_like(s["state"])
        return s
    N, G = case["N"], case["G"]
    xz = normal(B, L, 2 * C).to(T)
    bc = normal(B, L, 2 * G * N).to(T)
    s["x"], s["z"] = xz[..., :C], xz[..., C:]
    s["Bt"], s["Ct"] = (bc[..., i * G * N:(i + 1) * G * N].unflatten(2, (G, N)) for i in range(2))
    s["dt"], s["out"] = normal(B, L, C, std=0.5).to(T), torch.empty(B, L, C, device="cuda", dtype=T)
    s["A"] = -torch.arange(1, N + 1, device="cuda") * torch.exp(normal(C, N, std=0.1))
    s["D"] = normal(C, mean=1.0, std=0.2)
    s["dt_bias"] = torch.expm1(torch.exp(uniform(math.log(0.001), math.log(0.1), C))).log()
    if do == "step":
        for n in ("x", "z", "Bt", "Ct", "dt", "out"):
            s[n] = s[n][:, 0]
    if do == "step" or case["states"]:
        s["state"] = normal(B, C, N)
    if case["states"]:
        s["state_out"] = torch.empty_like(s["state"])
    if do == "train":
        s["d_out"] = normal(B, L, C).to(T)
        s["dxz"], s["dbc"] = (torch.zeros(B, L, n, device="cuda", dtype=T) for n in (2 * C, 2 * G * N))
        s["dx"], s["dz"] = s["dxz"][..., :C], s["dxz"][..., C:]
        s["dBt"], s["dCt"] = (s["dbc"][..., i * G * N:(i + 1) * G * N].unflatten(2, (G, N)) for i in range(2))
        s["ddt"] = torch.empty_like(s["dt"])
        for n in ("A", "D", "dt_bias"):
            s["d" + n] = torch.empty_like(s[n])
        if case["states"]:
            s["d_state_out"], s["d_state"] = normal(B, C, N), torch.empty_like(s["state"])
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _sigmoid(v):
    e = torch.exp(-v.abs())
    return torch.where(v >= 0, 1.0, e) / (1 + e)


def _softplus(v):
    return v.clamp(min=0) + torch.log1p(torch.exp(-v.abs()))


def _doubling(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, h in front of it zero: spans of 1, 2, 4 .. tokens are joined with those before them.  Overwrites both."""
    n, L = 1, a.shape[1]
    while n < L:
        b[:, n:] = b[:, n:] + a[:, n:] * b[:, :-n]
        a[:, n:] = a[:, n:] * a[:, :-n]
        n *= 2
    return b


def _plain_scan(s, grads):
    case = s["case"]
    B, L, C, N, G = (case[n] for n in ("B", "L", "C", "N", "G"))
    T, flip = s["x"].dtype, (lambda t: t.flip(1)) if case["reverse"] else (lambda t: t)
    x, dt, z, Bt, Ct = (flip(s[n].float()) for n in ("x", "dt", "z", "Bt", "Ct"))
    A, D = s["A"], s["D"]
    v = dt + s["dt_bias"]
    step = _softplus(v)
    split = lambda t: t.unflatten(2, (G, C // G))[..., None]   # noqa: E731  [B, L, G, C / G, 1]
    rows = lambda t: t[:, :, :, None]                          # noqa: E731  [B, L, G, 1, N]
    a = torch.exp(split(step) * A.view(G, C // G, N))
    h = split(step * x) * rows(Bt)
    if case["states"]:
        h[:, 0] += a[:, 0] * s["state"].view(B, G, C // G, N)
    h = _doubling(a.clone(), h)
    y = (h * rows(Ct)).sum(-1).flatten(2) + D * x
    sig = _sigmoid(z)
    gate = z * sig
    made = {"out": flip((y * gate).to(T))}
    if case["states"]:
        made["state_out"] = h[:, -1].reshape(B, C, N).clone()
    if not grads:
        return made
    do = flip(s["d_out"].float())
    dy = do * gate
    # g_t = C_t dy_t + a_{t+1} g_{t+1}, from the last token to the first
    g = rows(Ct) * split(dy)
    if case["states"]:
        g[:, -1] += s["d_state_out"].view(B, G, C // G, N)
    later = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1)
    g = _doubling(later.flip(1), g.flip(1)).flip(1)
    del later
    before = torch.zeros_like(h[:, :1]) if not case["states"] else s["state"].view(B, 1, G, C // G, N)
    through = g * a * torch.cat((before, h[:, :-1]), 1)     # what passes through a token's decay
    into = (g * rows(Bt)).sum(-1).flatten(2)
    dstep = (through * A.view(G, C // G, N)).sum(-1).flatten(2) + x * into
    dv = dstep * _sigmoid(v)
    made["dxz"] = torch.cat((flip((step * into + D * dy).to(T)), flip((do * y * sig * (1 + z * (1 - sig))).to(T))), 2)
    made["ddt"] = flip(dv.to(T))
    dB, dC = (g * split(step * x)).sum(3), (h * split(dy)).sum(3)
    made["dbc"] = torch.cat((flip(dB.flatten(2).to(T)), flip(dC.flatten(2).to(T))), 2)
    made["dA"] = (through * split(step)).sum((0, 1)).reshape(C, N)
    made["dD"], made["ddt_bias"] = (dy * x).sum((0, 1)), dv.sum((0, 1))
    if case["states"]:
        made["d_state"] = (a[:, 0] * g[:, 0]).reshape(B, C, N)
    return made


def _plain_step(s):
    case = s["case"]
    B, C, N, G = (case[n] for n in ("B", "C", "N", "G"))
    x, dt, z, Bt, Ct = (s[n].float() for n in ("x", "dt", "z", "Bt", "Ct"))
    step = _softplus(dt + s["dt_bias"])
    h = s["state"] * torch.exp(step[..., None] * s["A"])
    h = h.view(B, G, C // G, N) + (step * x).view(B, G, C // G, 1) * Bt[:, :, None]
    s["state"].copy_(h.view(B, C, N))
    y = (h * Ct[:, :, None]).sum(-1).view(B, C) + s["D"] * x
    return {"out": (y * z * _sigmoid(z)).to(s["x"].dtype), "state": s["state"]}


def _plain_conv(s, grads):
    case = s["case"]
    B, L, C, K = (case[n] for n in ("B", "L", "C", "K"))
    T, flip = s["x"].dtype, (lambda t: t.flip(1)) if case["reverse"] else (lambda t: t)
    w, x = s["weight"].float(), flip(s["x"].float())
    before = s["state"].float() if case["states"] else x.new_zeros(B, K - 1, C)
    x = torch.cat((before, x), 1)
    windows = x.unfold(1, K, 1)                                # [B, L, C, K]
    v = (windows * w).sum(-1) + s["bias"].float()
    sig = _sigmoid(v)
    made = {"out": flip((v * sig).to(T))}
    if case["states"]:
        made["state_out"] = x[:, L:].to(T)
    if grads:
        g = flip(s["d_out"].float()) * sig * (1 + v * (1 - sig))
        padded = torch.nn.functional.pad(g, (0, 0, K - 1, K - 1))
        dx = (padded.unfold(1, K, 1) * w.flip(1)).sum(-1)      # [B, L + K - 1, C], the window before the first token in front
        if case["states"]:
            dx[:, L:] += s["d_state_out"].float()
            made["d_state"] = dx[:, :K - 1].to(T)
        made["dx"] = flip(dx[:, K - 1:].to(T))
        made["dweight"], made["dbias"] = (windows * g[..., None]).sum((0, 1)).to(T), g.sum((0, 1)).to(T)
    return made


def _plain_conv_step(s):
    x = torch.cat((s["state"].float(), s["x"].float()[:, None]), 1)
    v = (x * s["weight"].float().t()).sum(1) + s["bias"].float()
    s["state"].copy_(x[:, 1:])
    return {"out": (v * _sigmoid(v)).to(s["x"].dtype), "state": s["state"]}


def _plain_norm(s, grads):
    case = s["case"]
    T, C = s["x"].dtype, case["C"]
    x, w = s["x"].float(), s["weight"].float()
    made = {}
    if case["residual"]:
        x = x + s["residual"].float()
        made["sum"] = x.to(T)
    rstd = 1 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    y = x * rstd * w
    if case["do"] == "norm8":
        blocks = torch.nn.functional.pad(y, (0, -C % 128)).unflatten(-1, (-1, 128)) if case["block"] else y[..., None, :]
        scales = (blocks.abs().amax(-1, keepdim=True) / 448).clamp(min=2.0 ** -126)
        made["out"] = (blocks / scales).flatten(-2)[..., :C].to(torch.float8_e4m3fn)
        made["scales"] = scales[..., 0]
        return made
    made["out"] = y.to(T)
    if grads:
        x = made["sum"].float() if case["residual"] else x      # as it was handed on
        gw = s["d_out"].float() * w
        dx = rstd * (gw - x * rstd.square() * (gw * x).mean(-1, keepdim=True))
        made["dx"] = (dx + s["d_sum"].float() if case["residual"] else dx).to(T)
        made["dweight"] = (s["d_out"].float() * x * rstd).sum((0, 1)).to(T)
    return made


def run(s):
    case = s["case"]
    do = case["do"]
    if not own:
        if do in ("norm", "norm8", "tnorm"):
            return _plain_norm(s, do == "tnorm")
        if do in ("conv", "tconv"):
            return _plain_conv(s, do == "tconv")
        if do == "cstep":
            return _plain_conv_step(s)
        return _plain_step(s) if do == "step" else _plain_scan(s, do == "train")
    import paper_2405_18425_b200 as vig

    get = s.get
    if do in ("norm", "norm8", "tnorm"):
        if do == "norm8":
            vig.vig_rms_norm_e4m3(s["x"], s["weight"], s["out"], s["scales"], residual=get("residual"), sum_out=get("sum"), eps=EPS)
            return {n: s[n] for n in ("sum", "out", "scales") if n in s}
        vig.vig_rms_norm(s["x"], s["weight"], s["out"], residual=get("residual"), sum_out=get("sum"), rstd=get("rstd"), eps=EPS)
        names = ["out", "sum"]
        if do == "tnorm":
            vig.vig_rms_norm_bwd(get("sum", s["x"]), s["weight"], s["rstd"], s["d_out"], s["dx"], s["dweight"], d_sum=get("d_sum"))
            names += ["dx", "dweight"]
        return {n: s[n] for n in names if n in s}
    if do == "cstep":
        vig.vig_causal_conv_step(s["x"], s["weight"], s["bias"], s["state"], s["out"], act="silu")
        return {n: s[n] for n in ("out", "state")}
    if do in ("conv", "tconv"):
        vig.vig_causal_conv(s["x"], s["weight"], s["bias"], s["out"], act="silu", state_in=get("state"), state_out=get("state_out"), reverse=case["reverse"])
        names = ["out", "state_out"]
        if do == "tconv":
            vig.vig_causal_conv_bwd(s["x"], s["weight"], s["bias"], s["d_out"], s["dx"], s["dweight"], s["dbias"], act="silu", state_in=get("state"),
                                    d_state_out=get("d_state_out"), d_state_in=get("d_state"), reverse=case["reverse"])
            names += ["dx", "dweight", "dbias", "d_state"]
        return {n: s[n] for n in names if n in s}
    x = [s[n] for n in ("x", "dt", "A", "Bt", "Ct")]
    more = {n: s[n] for n in ("D", "z", "dt_bias")}
    if do == "step":
        vig.vig_ssm_step(*x, s["state"], s["out"], **more)
        return {n: s[n] for n in ("out", "state")}
    vig.vig_ssm_fwd(*x, s["out"], **more, state_in=get("state"), state_out=get("state_out"), reverse=case["reverse"])
    names = ["out", "state_out"]
    if do == "train":
        vig.vig_ssm_bwd(*x, s["d_out"], *(s["d" + n] for n in ("x", "dt", "A", "Bt", "Ct")), **more, dD=s["dD"], dz=s["dz"], d_dt_bias=s["ddt_bias"],
                        state_in=get("state"), d_state_out=get("d_state_out"), d_state_in=get("d_state"), reverse=case["reverse"])
        names += ["dxz", "ddt", "dbc", "dA", "dD", "ddt_bias", "d_state"]
    return {n: s[n] for n in names if n in s}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------
def _exact_scan(s, grads):
    """Token by token; the gradient from the states of all tokens, kept, by the chain rule of one token."""
    case = s["case"]
    B, L, C, N, G = (case[n] for n in ("B", "L", "C", "N", "G"))
    x, dt, z = (s[n].double() for n in ("x", "dt", "z"))
    Bt, Ct = (s[n].double().repeat_interleave(C // G, 2) if G > 1 else s[n].double() for n in ("Bt", "Ct"))   # [B, L, C or 1, N]
    A, D = s["A"].double(), s["D"].double()
    v = dt + s["dt_bias"].double()
    step = torch.logaddexp(v, torch.zeros_like(v))
    h = s["state"].double() if case["states"] else x.new_zeros(B, C, N)
    order = range(L - 1, -1, -1) if case["reverse"] else range(L)
    y, kept = torch.empty_like(x), {}
    for t in order:
        if grads:
            kept[t] = h
        h = h * torch.exp(step[:, t, :, None] * A) + (step[:, t] * x[:, t])[..., None] * Bt[:, t]
        y[:, t] = (h * Ct[:, t]).sum(-1) + D * x[:, t]
    sig = torch.sigmoid(z)
    made = {"out": y * z * sig}
    if case["states"]:
        made["state_out"] = h
    if grads:
        do = s["d_out"].double()
        dy = do * z * sig
        dx, dstep = D * dy, torch.empty_like(x)
        dB, dC = (x.new_zeros(B, L, G, N) for _ in range(2))
        dA = torch.zeros_like(A)
        g = s["d_state_out"].double() if case["states"] else torch.zeros_like(h)
        per_group = lambda t: t.reshape(B, G, C // G, N).sum(2)   # noqa: E731
        for t in reversed(order):
            h = kept.pop(t)
            d, u = step[:, t, :, None], x[:, t, :, None]
            decay = torch.exp(d * A)
            new = h * decay + d * u * Bt[:, t]
            dC[:, t] = per_group(new * dy[:, t, :, None])
            g = g + Ct[:, t] * dy[:, t, :, None]
            dB[:, t] = per_group(g * d * u)
            dx[:, t] += (g * d * Bt[:, t]).sum(-1)
            g_decay = g * h * decay
            dA += (g_decay * d).sum(0)
            dstep[:, t] = (g_decay * A + g * u * Bt[:, t]).sum(-1)
            g = g * decay
        dv = dstep * torch.sigmoid(v)
        made.update(dxz=torch.cat((dx, do * y * (sig + z * sig * (1 - sig))), 2), ddt=dv, dbc=torch.cat((dB.flatten(2), dC.flatten(2)), 2), dA=dA,
                    dD=(dy * x).sum((0, 1)), ddt_bias=dv.sum((0, 1)))
        if case["states"]:
            made["d_state"] = g
    return made


def _exact_conv(s, grads):
    case = s["case"]
    B, L, C, K = (case[n] for n in ("B", "L", "C", "K"))
    w = s["weight"].double()
    at = lambda t: L - 1 - t if case["reverse"] else t   # noqa: E731
    past = s["state"].double() if case["states"] else w.new_zeros(B, K - 1, C)
    order = torch.tensor([at(t) for t in range(L)], device="cuda")
    line = torch.cat((past, s["x"].double()[:, order]), 1)
    v = s["bias"].double().expand(B, L, C).clone()
    for k in range(K):
        v += line[:, k:k + L] * w[:, k]
    sig = torch.sigmoid(v)
    made = {"out": (v * sig)[:, order]}      # (the order is its own inverse)
    if case["states"]:
        made["state_out"] = line[:, L:]
    if grads:
        g = s["d_out"].double()[:, order] * (sig + v * sig * (1 - sig))
        dline, dw = torch.zeros_like(line), torch.empty_like(w)
        for k in range(K):
            dline[:, k:k + L] += g * w[:, k]
            dw[:, k] = (g * line[:, k:k + L]).sum((0, 1))
        if case["states"]:
            dline[:, L:] += s["d_state_out"].double()
            made["d_state"] = dline[:, :K - 1]
        made.update(dx=dline[:, K - 1:][:, order], dweight=dw, dbias=g.sum((0, 1)))
    return made


def _exact_norm(s, grads):
    case = s["case"]
    w = s["weight"].double()
    x = s["x"].double()
    made = {}
    if case["residual"]:
        x = x + s["residual"].double()
        made["sum"] = x
    rstd = (x.pow(2).sum(-1, keepdim=True) / case["C"] + EPS).rsqrt()
    y = x * rstd * w
    if case["do"] == "norm8":
        pieces = y.split(128 if case["block"] else case["C"], -1)
        scales = [p.abs().max(-1, keepdim=True).values / 448 for p in pieces]
        made["out"] = torch.cat([(p / c).to(torch.float8_e4m3fn).double() for p, c in zip(pieces, scales)], -1)
        made["scales"] = torch.cat(scales, -1)
        return made
    made["out"] = y
    if grads:
        if case["residual"]:
            x = x.to(s["x"].dtype).double()      # as it was handed on
        do = s["d_out"].double()
        dx = do * w * rstd - x * rstd.pow(3) * (do * w * x).sum(-1, keepdim=True) / case["C"]
        made["dx"] = dx + s["d_sum"].double() if case["residual"] else dx
        made["dweight"] = (do * x * rstd).sum((0, 1))
    return made


def exact(case, seed):
    s = prepare(case, seed)
    do = case["do"]
    if do in ("norm", "norm8", "tnorm"):
        return _exact_norm(s, do == "tnorm")
    if do in ("conv", "tconv"):
        return _exact_conv(s, do == "tconv")
    if do == "cstep":
        line = torch.cat((s["state"], s["x"][:, None]), 1).double()
        v = torch.einsum("bkc,ck->bc", line, s["weight"].double()) + s["bias"].double()
        return {"out": v * torch.sigmoid(v), "state": line[:, 1:]}
    if do == "step":
        C, G = case["C"], case["G"]
        x, dt, z, Bt, Ct, A, h = (s[n].double() for n in ("x", "dt", "z", "Bt", "Ct", "A", "state"))
        v = dt + s["dt_bias"].double()
        d = torch.logaddexp(v, torch.zeros_like(v))
        h = h * torch.exp(torch.einsum("bc,cn->bcn", d, A)) + torch.einsum("bc,bcn->bcn", d * x, Bt.repeat_interleave(C // G, 1))
        y = torch.einsum("bcn,bcn->bc", h, Ct.repeat_interleave(C // G, 1)) + s["D"].double() * x
        return {"out": y * z * torch.sigmoid(z), "state": h}
    return _exact_scan(s, do == "train")


def work(case):
    """Each input read once, each output written once; the arithmetic of a state and token (decay, input, read-out; with the gradient the
    adjoint's and the five sums over it), a logarithm or an exponential counted as one operation."""
    do, e = case["do"], 2 if case["dtype"] == "bf16" else 4
    B, L, C = (case[n] for n in ("B", "L", "C"))
    n = B * L * C
    if do in ("norm", "norm8", "tnorm"):
        r = 2 if case["residual"] else 0
        if do == "norm8":
            return {"bytes": (1 + r) * n * e + n + B * L * (-(-C // 128) if case["block"] else 1) * 4 + C * e, "flops": 6 * n}
        if do == "norm":
            return {"bytes": (2 + r) * n * e + C * e, "flops": 4 * n}
        # sum and rstd stay in hand between the two calls' work
        return {"bytes": (2 + r) * n * e + (2 + r // 2) * n * e + 2 * C * e, "flops": 14 * n}
    if do == "cstep":
        return {"bytes": (2 + 2 * (case["K"] - 1)) * n * e + (case["K"] + 1) * C * e, "flops": (2 * case["K"] + 4) * n}
    if do in ("conv", "tconv"):
        state = B * (case["K"] - 1) * C * e if case["states"] else 0
        if do == "conv":
            return {"bytes": 2 * n * e + 2 * state + (case["K"] + 1) * C * e, "flops": (2 * case["K"] + 4) * n}
        return {"bytes": 4 * n * e + 4 * state + 2 * (case["K"] + 1) * C * e, "flops": (6 * case["K"] + 12) * n}
    N, G = case["N"], case["G"]
    rows, params, state = 2 * B * L * G * N * e, 4 * (C * N + 2 * C), 4 * B * C * N
    if do == "step":
        return {"bytes": 4 * n * e + rows + params + 2 * state, "flops": 7 * n * N}
    if do == "scan":
        return {"bytes": 4 * n * e + rows + params + (2 * state if case["states"] else 0), "flops": 7 * n * N}
    return {"bytes": 8 * n * e + 2 * rows + 2 * params + (4 * state if case["states"] else 0), "flops": 25 * n * N}
