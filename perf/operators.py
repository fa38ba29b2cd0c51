"""Timing cases of what a training step needs around the layer: the gated feed-forward block and its
gradients, the norms around a residual sum and their gradients, and the update of the weights.

A case is one call.  `run` computes it in plain torch operations (32-bit arithmetic, rounded once at
the end) or, with `own`, through the framework's entry points.  Sizes: the stage maps of
synthetic_inputs.py, the channel counts of perf/cases.py, and generic ones up to 1024 channels.  A gated
block of hidden = 2 C has the parameters of the ungated one with expansion 3, hidden = 8/3 C those of
expansion 4.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
EPS = 1e-6          # of the norms
BLOCK = 32          # values that share a scale in 8-bit optimizer states


def ffn(name, op, dtype, M, C, hidden, act, bias, pre):
    """op "ffn" or "ffn_bwd"; pre: the forward hands its pre-activations to the caller, the backward is given them."""
    return dict(name=name, op=op, dtype=dtype, M=M, C=C, hidden=hidden, act=act, bias=bias, pre=pre)


def norm(name, op, dtype, groups, rows, C, kind, post, gate):
    """op "norm" or "norm_bwd"; groups x rows tokens, a row of the gate for each group where there is one."""
    return dict(name=name, op=op, dtype=dtype, groups=groups, rows=rows, C=C, kind=kind, post=post, gate=gate)


def adamw(name, bits, dtype, grad, copies, layers, C, hidden):
    """The tensors of `layers` blocks: Wqkv, Wo, Wlce, W1, b1, W2, b2 and two norms each."""
    return dict(name=name, op="adamw", bits=bits, dtype=dtype, grad=grad, copies=copies, layers=layers, C=C, hidden=hidden)


def listed():
    return [
        # one token through a block of the plain-ViT width: latency, and every weight read once
        ffn("ffn_one_token", "ffn", "bf16", 1, 768, 2048, "silu", False, False),
        # a classification batch at the third stage, as it is served
        ffn("ffn_stage3_b64", "ffn", "bf16", 64 * 14 * 14, 256, 512, "gelu", True, False),
        # the forward of a training step on a wide model, which keeps the pre-activations
        ffn("ffn_train_wide", "ffn", "bf16", 32768, 1024, 2816, "silu", False, True),
        # its gradients
        ffn("ffn_bwd_wide", "ffn_bwd", "bf16", 16384, 1024, 2816, "silu", False, True),
        # gradients at the second stage, pre-activations formed again
        ffn("ffn_bwd_stage2_b16", "ffn_bwd", "bf16", 16 * 28 * 28, 128, 256, "gelu", True, False),
        # float32 gradients at sizes that nothing divides (a cropped map, an odd width)
        ffn("ffn_bwd_odd_f32", "ffn_bwd", "f32", 3 * 23 * 29, 99, 261, "silu", True, False),
        # one token between two halves of a block
        norm("norm_one_token", "norm", "bf16", 1, 1, 768, "rms", False, False),
        # a classification batch at the first stage: both norms, residual scale and a gate per image
        norm("norm_stage1_b64", "norm", "bf16", 64, 56 * 56, 64, "layer", True, True),
        # gradients of the same on a training batch of the plain ViT
        norm("norm_bwd_vit_b32", "norm_bwd", "bf16", 32, 32 * 32, 768, "layer", True, True),
        # float32 gradients of the plain pre-norm form, odd rows
        norm("norm_bwd_f32", "norm_bwd", "f32", 5, 35 * 37, 192, "rms", False, False),
        # one block's tensors, states in 32 bits: a launch's latency
        adamw("adamw_block", 32, "f32", "f32", False, 1, 64, 128),
        # a deep model's tensors, states in 8 bits, float32 weights with the bf16 copies that the forward reads
        adamw("adamw_model_8bit", 8, "f32", "bf16", True, 18, 512, 1365),
    ]


CHANNELS = (64, 96, 128, 192, 256, 384, 512, 768, 1024)


def _cost(c):
    """Rough cost in bytes moved: products at their types' rates."""
    w = work(c)
    rate = 12 if c.get("dtype") == "f32" else 200
    return max(w["bytes"], w["flops"] / rate)


def draw(rng):
    log = lambda lo, hi: int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["ffn", "ffn", "ffn", "ffn_bwd", "ffn_bwd", "norm", "norm", "norm_bwd", "norm_bwd", "adamw"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        C = rng.choice(CHANNELS) if rng.random() < 0.8 else log(16, 1024)
        if op in ("ffn", "ffn_bwd"):
            hidden = int(C * rng.uniform(1.0, 4.0))
            step = rng.choice([1, 8, 32, 64])
            hidden = max(step, hidden // step * step)
            c = ffn("", op, dtype, log(1 if op == "ffn" else 16, 32768), C, hidden, rng.choice(["silu", "gelu"]), rng.random() < 0.5, rng.random() < 0.5)
        elif op in ("norm", "norm_bwd"):
            tokens = log(1, 262144)
            groups = min(tokens, rng.choice([1, log(1, 64), log(1, 64), log(1, 262144)]))
            c = norm("", op, dtype, groups, max(1, tokens // groups), C, rng.choice(["layer", "rms"]), rng.random() < 0.5, rng.random() < 0.6)
        else:
            c = adamw("", rng.choice([8, 32]), rng.choice(["f32", "f32", "bf16"]), rng.choice(["f32", "bf16"]), rng.random() < 0.5, log(1, 24), C,
                      int(C * rng.uniform(1.0, 4.0)))
            if c["dtype"] == "bf16":
                c["copies"] = False
        del c["name"]
        if _cost(c) <= most:
            return c


def _tensor_sizes(c):
    C, h = c["C"], c["hidden"]
    return [C * 3 * C, C * C, C * 25, C * 2 * h, 2 * h, h * C, C, C, C, C, C] * c["layers"]


def _places(sizes):
    """Where each tensor's values begin in flat buffers of whole blocks, and the buffers' length."""
    at, places = 0, []
    for n in sizes:
        places.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return places, at


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    if c["op"] in ("ffn", "ffn_bwd"):
        dt, M, C, h = DTYPES[c["dtype"]], c["M"], c["C"], c["hidden"]
        s = dict(c, X=randn(M, C).to(dt), W1=(randn(C, 2 * h) / C ** 0.5).to(dt), W2=(randn(h, C) / h ** 0.5).to(dt),
                 b1=0.1 * randn(2 * h) if c["bias"] else None, b2=0.1 * randn(C) if c["bias"] else None)
        if c["op"] == "ffn_bwd":
            s["dY"] = randn(M, C).to(dt)
            s["saved"] = _pre(s["X"].float(), s["W1"].float(), s["b1"]).to(dt) if c["pre"] else None
        return s
    if c["op"] in ("norm", "norm_bwd"):
        dt, G, n, C = DTYPES[c["dtype"]], c["groups"], c["rows"], c["C"]
        vec = lambda mean, dev: mean + dev * randn(C)
        # a residual stream with an offset per channel, as a network's has
        s = dict(c, X=(randn(G, n, C) + 0.5 * randn(C)).to(dt), Y=randn(G, n, C).to(dt), gamma=vec(1.0, 0.1), beta=vec(0.0, 0.1),
                 scale=vec(0.5, 0.1), post_gamma=vec(1.0, 0.1) if c["post"] else None, post_beta=vec(0.0, 0.1) if c["post"] else None,
                 gate=randn(G, C).to(dt) if c["gate"] else None)
        if c["op"] == "norm_bwd":
            s.update(dN=randn(G, n, C).to(dt), dX=randn(G, n, C).to(dt))
        return s
    sizes = _tensor_sizes(c)
    places, total = _places(sizes)
    # the model's weights, gradients and bf16 copies each in one buffer, a view for every tensor
    cut = lambda flat: [flat[a:a + n] for a, n in zip(places, sizes)]
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    for a, n in zip(places, sizes):
        live[a:a + n] = True
    noise = lambda: torch.where(live, randn(total) * torch.exp(1.5 * randn(total)), 0.0)    # heavy tails
    weights, grads = (0.02 * torch.where(live, randn(total), 0.0)).to(DTYPES[c["dtype"]]), (1e-3 * noise()).to(DTYPES[c["grad"]])
    m, r = 1e-3 * noise(), 1e-3 * noise().abs()
    s = dict(c, weights=weights, grads=grads, W=cut(weights), dW=cut(grads))
    if c["bits"] == 32:
        s["state"] = {"exp_avg": m, "exp_avg_sq": r * r}
    else:
        (mc, ms), (rc, rs) = _encode(m, False), _encode(r, True)
        s["state"] = {"exp_avg": mc, "exp_avg_scale": ms, "exp_avg_root": rc, "exp_avg_root_scale": rs}
    s["copy"] = weights.to(torch.bfloat16) if c["copies"] else None
    s["copied"] = cut(s["copy"]) if c["copies"] else None
    return s


# -- plain forms -------------------------------------------------------------------------------------------------

def _pre(X, W1, b1):
    P = X @ W1
    return P if b1 is None else P + b1


def _act(G, act):
    """The activation and its derivative."""
    if act == "silu":
        s = 1 / (1 + torch.exp(-G))
        return G * s, s * (1 + G * (1 - s))
    cdf = 0.5 * (1 + torch.erf(G * 0.5 ** 0.5))
    return G * cdf, cdf + G * torch.exp(-0.5 * G * G) * (0.5 / math.pi) ** 0.5


def _ffn(s, f):
    """f: the type of the arithmetic."""
    X, W1, W2 = s["X"].to(f), s["W1"].to(f), s["W2"].to(f)
    b1, b2, h = (None if s["b1"] is None else s["b1"].to(f)), (None if s["b2"] is None else s["b2"].to(f)), s["hidden"]
    if s["op"] == "ffn":
        P = _pre(X, W1, b1)
        Y = (_act(P[:, :h], s["act"])[0] * P[:, h:]) @ W2
        if b2 is not None:
            Y = Y + b2
        return [Y, P] if s["pre"] else [Y]
    dY = s["dY"].to(f)
    P = s["saved"].to(f) if s["pre"] else _pre(X, W1, b1)
    a, slope = _act(P[:, :h], s["act"])
    U, dA = P[:, h:], dY @ W2.t()
    dP = torch.cat([dA * U * slope, dA * a], dim=1)
    out = [dP @ W1.t(), X.t() @ dP, (a * U).t() @ dY]
    return out + [dP.sum(0), dY.sum(0)] if s["bias"] else out


def _unit(X, kind):
    """X over its norm, and one over that."""
    if kind == "layer":
        X = X - X.mean(-1, keepdim=True)
    inv = 1 / torch.sqrt((X * X).mean(-1, keepdim=True) + EPS)
    return X * inv, inv


def _unit_bwd(dU, U, inv, kind):
    d = dU - U * (dU * U).mean(-1, keepdim=True)
    return inv * (d - dU.mean(-1, keepdim=True) if kind == "layer" else d)


def _norm(s, f):
    vec = lambda k: None if s[k] is None else s[k].to(f)
    X, Y, gamma, beta, scale, pg, pb = s["X"].to(f), s["Y"].to(f), vec("gamma"), vec("beta"), vec("scale"), vec("post_gamma"), vec("post_beta")
    kind, gate = s["kind"], 1.0 if s["gate"] is None else s["gate"].to(f)[:, None, :]
    if s["post"]:
        yu, yinv = _unit(Y, kind)
        Z = yu * pg + pb
    else:
        Z = Y
    if s["op"] == "norm":
        R = X + scale * gate * Z
        return [R, _unit(R, kind)[0] * gamma + beta]
    # X is the sum that the forward returned
    dN, u = s["dN"].to(f), None
    u, inv = _unit(X, kind)
    D = s["dX"].to(f) + _unit_bwd(dN * gamma, u, inv, kind)
    dZ = D * scale * gate
    rows = lambda t: t.sum((0, 1))
    out = {"dX": D, "dgamma": rows(dN * u), "dbeta": rows(dN), "dscale": rows(D * gate * Z)}
    if s["gate"] is not None:
        out["dgate"] = (D * scale * Z).sum(1)
    if s["post"]:
        out["dpost_gamma"], out["dpost_beta"] = rows(dZ * yu), rows(dZ)
        dZ = _unit_bwd(dZ * pg, yu, yinv, kind)
    out["dY"] = dZ
    return out


STEP, LR, BETA1, BETA2, ADAM_EPS, DECAY = 11, 1e-3, 0.9, 0.999, 1e-8, 0.05


def _encode(x, root):
    """Codes (e4m3) and scales (powers of two) of blocks of 32 values: the smallest scale with which the largest value is at most
    448.  A root that is not zero keeps the smallest code at least."""
    x = x.view(-1, BLOCK)
    m, e = torch.frexp(x.abs().amax(1, keepdim=True))
    e = torch.clamp(e - 9 + (m > 0.875).to(torch.int32), min=-126)
    codes = torch.ldexp(x, -e).to(torch.float32)
    if root:
        codes = torch.where((codes > 0) & (codes < 2.0 ** -9), 2.0 ** -9, codes)
    scales = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu).view(-1)
    return codes.to(torch.float8_e4m3fn).view(-1), scales


def _decode(codes, scales, f):
    e = scales.view(torch.uint8).to(torch.int32) - 127
    return torch.ldexp(codes.to(f).view(-1, BLOCK), e[:, None]).view(-1)


def _adamw(s, f):
    """New weights and states.  The scalars of the step are float32 numbers, as its arithmetic takes them."""
    st = s["state"]
    as32 = lambda v: torch.tensor(v, dtype=torch.float32).item()
    p, g = s["weights"].to(f), s["grads"].to(f)
    if s["bits"] == 32:
        m, v = st["exp_avg"].to(f), st["exp_avg_sq"].to(f)
    else:
        m, r = _decode(st["exp_avg"], st["exp_avg_scale"], f), _decode(st["exp_avg_root"], st["exp_avg_root_scale"], f)
        v = r * r
    m = as32(BETA1) * m + as32(1 - BETA1) * g
    v = as32(BETA2) * v + as32(1 - BETA2) * (g * g)
    root = torch.sqrt(v)
    p = p * as32(1 - LR * DECAY) - as32(LR / (1 - BETA1 ** STEP)) * (m / (root * as32(1 / math.sqrt(1 - BETA2 ** STEP)) + as32(ADAM_EPS)))
    return p, m, v, root


def _adamw_out(s, weights, state, copy):
    return [weights] + [state[k] for k in sorted(state)] + ([copy] if s["copies"] else [])


def _adamw_plain(s, f=torch.float32, keep=True):
    p, m, v, root = _adamw(s, f)
    weights = p.to(DTYPES[s["dtype"]]) if keep else p
    copy = weights.to(torch.bfloat16) if s["copies"] and keep else p
    if s["bits"] == 32:
        state = {"exp_avg": m, "exp_avg_sq": v}
    else:
        (mc, ms), (rc, rs) = _encode(m, False), _encode(root, True)
        state = {"exp_avg": mc, "exp_avg_scale": ms, "exp_avg_root": rc, "exp_avg_root_scale": rs}
    if not keep:
        return _adamw_out(s, weights, state, copy)
    s["weights"].copy_(weights)
    for k in state:
        s["state"][k].copy_(state[k])
    if s["copies"]:
        s["copy"].copy_(copy)
    return _adamw_out(s, s["weights"], s["state"], s["copy"])


def _round(out, s):
    """The plain form's 32-bit results in the types that the operators return."""
    dt = DTYPES[s["dtype"]]
    if isinstance(out, dict):
        return {k: v.to(dt) if k in ("dX", "dY", "dgate") else v for k, v in out.items()}
    return [v.to(dt) for v in out]


def run(s):
    if not own:
        if s["op"] == "adamw":
            return _adamw_plain(s)
        f = torch.float32
        return _round(_ffn(s, f) if s["op"] in ("ffn", "ffn_bwd") else _norm(s, f), s)
    import paper_2303_08810_amd as bra
    if s["op"] == "ffn":
        out = bra.bra_ffn_forward(s["X"], s["W1"], s["W2"], b1=s["b1"], b2=s["b2"], act=s["act"], want_pre=s["pre"])
        return list(out) if s["pre"] else [out]
    if s["op"] == "ffn_bwd":
        return list(bra.bra_ffn_backward(s["X"], s["W1"], s["W2"], s["dY"], b1=s["b1"], pre=s["saved"], act=s["act"], bias_grads=s["bias"]))
    args = {k: s[k] for k in ("post_gamma", "post_beta", "scale", "gate", "kind")} if "kind" in s else {}
    if s["op"] == "norm":
        return list(bra.bra_norm_forward(s["X"], s["gamma"], s["beta"], Y=s["Y"], eps=EPS, **args))
    if s["op"] == "norm_bwd":
        return bra.bra_norm_backward(s["X"], s["gamma"], s["dN"], dX=s["dX"], Y=s["Y"], eps=EPS, **args)
    bra.bra_adamw_step(s["W"], s["dW"], s["state"], step=STEP, lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY, copies=s["copied"])
    return _adamw_out(s, s["weights"], s["state"], s["copy"])


def work(c):
    if c["op"] in ("ffn", "ffn_bwd"):
        M, C, h, b = c["M"], c["C"], c["hidden"], BYTES[c["dtype"]]
        weights, product = 3 * C * h, 2.0 * M * C * h
        if c["op"] == "ffn":
            return {"bytes": b * (2 * M * C + weights + (2 * M * h if c["pre"] else 0)), "flops": 3 * product}
        return {"bytes": b * (3 * M * C + weights + (2 * M * h if c["pre"] else 0)) + 4 * weights, "flops": (6 if c["pre"] else 8) * product}
    if c["op"] in ("norm", "norm_bwd"):
        n, b = c["groups"] * c["rows"] * c["C"], BYTES[c["dtype"]]
        gate = c["groups"] * c["C"] * b if c["gate"] else 0
        if c["op"] == "norm":
            return {"bytes": 4 * n * b + gate, "flops": 16.0 * n}
        return {"bytes": 6 * n * b + 2 * gate, "flops": 40.0 * n}
    n = sum(_tensor_sizes(c))
    state = 16 if c["bits"] == 32 else 4 + 4 / BLOCK
    return {"bytes": n * (2 * BYTES[c["dtype"]] + BYTES[c["grad"]] + state + (2 if c["copies"] else 0)), "flops": 16.0 * n}


# -- in 64 bits, from the definitions ----------------------------------------------------------------------------

def _wide(s):
    return {k: v.double() if isinstance(v, torch.Tensor) and v.dtype in (torch.float32, torch.bfloat16) else v for k, v in s.items()}


def _exact_ffn(c, s):
    h, phi = c["hidden"], torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device="cuda"), 1.0, validate_args=False)
    cdf = torch.sigmoid if c["act"] == "silu" else phi.cdf
    if c["op"] == "ffn" or not c["pre"]:
        G, U = s["X"].matmul(s["W1"][:, :h]), s["X"].matmul(s["W1"][:, h:])
        if c["bias"]:
            G, U = G + s["b1"][:h], U + s["b1"][h:]
    else:
        G, U = s["saved"].split(h, dim=1)
    q = cdf(G)
    if c["op"] == "ffn":
        Y = (G * q * U).matmul(s["W2"])
        Y = Y + s["b2"] if c["bias"] else Y
        return [Y, torch.cat([G, U], 1)] if c["pre"] else [Y]
    density = q * (1 - q) if c["act"] == "silu" else torch.exp(phi.log_prob(G))
    dA = s["dY"].matmul(s["W2"].t().contiguous())
    dG, dU = dA * U * (q + G * density), dA * G * q
    dX = dG.matmul(s["W1"][:, :h].t().contiguous()) + dU.matmul(s["W1"][:, h:].t().contiguous())
    Xt = s["X"].t().contiguous()
    out = [dX, torch.cat([Xt.matmul(dG), Xt.matmul(dU)], 1), (G * q * U).t().contiguous().matmul(s["dY"])]
    return out + [torch.cat([dG.sum(0), dU.sum(0)]), s["dY"].sum(0)] if c["bias"] else out


def _exact_norm(c, s):
    """The gradients by automatic differentiation of the sum of products with what comes in."""
    def rule(x, weight, bias):
        mid = x.mean(-1, keepdim=True) if c["kind"] == "layer" else torch.zeros_like(x[..., :1])
        spread = ((x - mid) ** 2).sum(-1, keepdim=True) / c["C"]
        return (x - mid) / (spread + EPS).sqrt() * weight + bias

    def branch(Y, pg, pb, scale, gate):
        Z = rule(Y, pg, pb) if c["post"] else Y
        Z = Z * scale
        return Z * gate.unsqueeze(1) if c["gate"] else Z

    if c["op"] == "norm":
        R = s["X"] + branch(s["Y"], s["post_gamma"], s["post_beta"], s["scale"], s["gate"])
        return [R, rule(R, s["gamma"], s["beta"])]
    live = {k: s[k].clone().requires_grad_() for k in ("X", "Y", "gamma", "beta", "scale", "gate", "post_gamma", "post_beta") if s[k] is not None}
    get = lambda k: live.get(k)
    # the sum's own gradient first, then the branch's from it
    dR, dgamma, dbeta = torch.autograd.grad((rule(live["X"], live["gamma"], live["beta"]) * s["dN"]).sum() + (live["X"] * s["dX"]).sum(),
                                            [live["X"], live["gamma"], live["beta"]])
    names = [k for k in ("Y", "scale", "gate", "post_gamma", "post_beta") if k in live]
    grads = torch.autograd.grad((branch(live["Y"], get("post_gamma"), get("post_beta"), live["scale"], get("gate")) * dR).sum(), [live[k] for k in names])
    return {"dX": dR, "dgamma": dgamma, "dbeta": dbeta, **{"d" + k: t for k, t in zip(names, grads)}}


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] in ("ffn", "ffn_bwd"):
        return _exact_ffn(c, _wide(s))
    if c["op"] in ("norm", "norm_bwd"):
        return _exact_norm(c, _wide(s))
    st, f = s["state"], torch.float64
    p, g = s["weights"].to(f), s["grads"].to(f)
    number = lambda v: float(torch.tensor(v, dtype=torch.float32))
    if c["bits"] == 32:
        m, v = st["exp_avg"].to(f), st["exp_avg_sq"].to(f)
    else:
        lift = lambda codes, scales: (codes.to(f).view(-1, BLOCK) * torch.exp2(scales.view(torch.uint8).to(f) - 127)[:, None]).view(-1)
        m, v = lift(st["exp_avg"], st["exp_avg_scale"]), lift(st["exp_avg_root"], st["exp_avg_root_scale"]).square()
    m, v = m.lerp(g, number(1 - BETA1)), v * number(BETA2) + g.square() * number(1 - BETA2)
    away = m * number(LR / (1 - BETA1 ** STEP)) / (v.sqrt() * number(1 / math.sqrt(1 - BETA2 ** STEP)) + number(ADAM_EPS))
    p = p * number(1 - LR * DECAY) - away
    if c["bits"] == 32:
        state = [m, v]
    else:
        def codes(x, root):
            x = x.view(-1, BLOCK)
            top = x.abs().amax(1)
            e = torch.ceil(torch.log2(top / 448).clamp(min=-126.0))      # the smallest power of two that takes the largest value to 448
            q = x * torch.exp2(-e)[:, None]
            if root:
                q = torch.where(x > 0, q.clamp(min=2.0 ** -9), q)
            return q.float().to(torch.float8_e4m3fn).view(-1), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
        (mc, ms), (rc, rs) = codes(m, False), codes(v.sqrt(), True)
        state = [mc, rc, rs, ms]        # as run() has them, in the order of their names
    return [p] + state + ([p] if c["copies"] else [])
