"""Timing cases of attention between whole sequences: the norms and the position rotation of queries and keys with
their gradients, attention and its gradients.

A case is one call.  `run` computes it in plain torch operations (32-bit arithmetic, rounded once at
the end) or, with `own`, through the framework's entry points.  Sizes: the last stage and the plain-ViT adaptation of
synthetic_inputs.py, and generic ones with heads of up to 128 channels.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
EPS = 1e-6          # of the norms
BASE = 10000.0      # of the rotation's angles


def qk(name, op, dtype, B, N, heads, kv, d, norm, turned, pairs, far):
    """op "qk" or "qk_bwd"; turned: channels of a head that are rotated; far: the sequences begin at positions of their own, up to this one."""
    return dict(name=name, op=op, dtype=dtype, B=B, N=N, heads=heads, kv=kv, d=d, norm=norm, turned=turned, pairs=pairs, far=far)


def att(name, op, dtype, B, Nq, Nk, heads, kv, d, causal, q_ragged, k_ragged, where, lse):
    """op "att" or "att_bwd"; where: "packed" (queries, keys and values side by side in one buffer), "cache" (keys and values [B, kv, Nk, d]) or
    "apart"; ragged: sequences of lengths from 1 / B of it to the whole; lse: the forward returns what its gradients need."""
    return dict(name=name, op=op, dtype=dtype, B=B, Nq=Nq, Nk=Nk, heads=heads, kv=kv, d=d, causal=causal, q_ragged=q_ragged, k_ragged=k_ragged, where=where, lse=lse)


def listed():
    return [
        # one token's queries and keys at the plain-ViT width, as a token is added to a cache: latency
        qk("qk_one_token", "qk", "bf16", 1, 1, 12, 12, 64, True, 64, "halves", 4096),
        # a training batch of the plain-ViT adaptation, out of the projection's buffer
        qk("qk_vit_b32", "qk", "bf16", 32, 1024, 12, 12, 64, True, 64, "halves", 0),
        # gradients of long sequences with shared keys, half of the channels rotated in neighbouring pairs
        qk("qk_bwd_long", "qk_bwd", "bf16", 2, 8192, 32, 8, 128, True, 64, "neighbours", 0),
        # float32 gradients at a cropped map's size and an odd width
        qk("qk_bwd_odd_f32", "qk_bwd", "f32", 5, 35 * 37, 6, 6, 40, True, 40, "halves", 0),
        # the next token of one short sequence, as it is served: latency
        att("att_one_token", "att", "bf16", 1, 1, 197, 12, 12, 64, False, False, False, "cache", False),
        # the next token of 8 sequences of up to 32768: keys and values read once
        att("att_one_token_long", "att", "bf16", 8, 1, 32768, 32, 8, 128, False, False, True, "cache", False),
        # the plain-ViT adaptation, a training batch with attention over the whole map
        att("att_vit_b32", "att", "bf16", 32, 1024, 1024, 12, 12, 64, False, False, False, "packed", True),
        # a long causal sequence with shared keys
        att("att_long_causal", "att", "bf16", 1, 8192, 8192, 32, 8, 128, True, False, False, "packed", True),
        # float32, a padded batch of odd maps, heads that no tile divides
        att("att_odd_f32", "att", "f32", 3, 23 * 29, 23 * 29, 6, 6, 40, False, True, True, "packed", False),
        # gradients of the last stage, where each token attends to the whole 7 x 7 map
        att("att_bwd_stage4_b64", "att_bwd", "bf16", 64, 49, 49, 16, 16, 32, False, False, False, "packed", True),
        # gradients of a long causal sequence with shared keys
        att("att_bwd_long_causal", "att_bwd", "bf16", 1, 8192, 8192, 16, 4, 128, True, False, False, "packed", True),
        # float32 gradients, padded causal batch, shared keys, odd sizes
        att("att_bwd_odd_f32", "att_bwd", "f32", 2, 35 * 37, 35 * 37, 8, 2, 72, True, True, True, "apart", True),
    ]


def _cost(c):
    """Rough cost: of products in multiply-adds, of passes over memory in bytes at the same rate."""
    w = work(c)
    if c["op"] in ("qk", "qk_bwd"):
        return 100 * w["bytes"]
    pairs = c["B"] * c["heads"] * c["Nq"] * c["Nk"]
    return max(100 * w["bytes"], pairs * (c["d"] + 64) * (2.5 if c["op"] == "att_bwd" else 1) * (8 if c["dtype"] == "f32" else 1))


def draw(rng):
    log = lambda lo, hi: min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999)))))
    # the longest of the listed passes over memory for the first kind, the most expensive case for the second
    most = {kind: max(_cost(c) for c in listed() if c["op"].startswith(kind)) for kind in ("qk", "att")}
    while True:
        op = rng.choice(["qk", "qk", "qk_bwd", "qk_bwd", "att", "att", "att", "att", "att_bwd", "att_bwd", "att_bwd"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([32, 64, 64, 128, 128]) if rng.random() < 0.7 else 8 * rng.randint(2, 16)
        kv = log(1, 16)
        heads = kv * rng.choice([1, 1, 2, 4, 8, rng.randint(1, 7)])
        if heads > 48:
            continue
        if op in ("qk", "qk_bwd"):
            tokens = log(1, 65536)
            B = log(1, min(tokens, 64))
            turned = rng.choice([d, d, d, d // 2 // 2 * 2, 0])
            norm = rng.random() < 0.8 or not turned
            c = qk("", op, dtype, B, max(1, tokens // B), heads, kv, d, norm, turned, rng.choice(["halves", "neighbours"]), rng.choice([0, 0, log(1, 131072)]))
        else:
            form = rng.choice(["self", "self", "self", "chunk", "cross"] + (["one", "one"] if op == "att" else []))
            B = log(1, 64)
            if form == "self":
                Nq = Nk = log(1, 8192)
            elif form == "one":
                Nq, Nk = 1, log(1, 65536)
            else:
                Nq, Nk = log(1, 2048), log(1, 16384)
                if form == "chunk" and Nq > Nk:
                    continue
            ragged = B > 1 and rng.random() < 0.3
            c = att("", op, dtype, B, Nq, Nk, heads, kv, d, form == "chunk" or (form == "self" and rng.random() < 0.5), ragged and form == "self", ragged,
                    "packed" if form == "self" and rng.random() < 0.7 else rng.choice(["cache", "apart"]), op == "att_bwd" or rng.random() < 0.3)
        del c["name"]
        if _cost(c) <= most[op.split("_")[0]]:
            return c


# -- inputs ------------------------------------------------------------------------------------------------------

def _lengths(n, B):
    """From 1 / B of n to n."""
    return [max(1, n * (b + 1) // B) for b in range(B)]


def _table(T, turned):
    """Cosines and sines of the rotation, as a program makes them once."""
    angle = torch.arange(T, dtype=torch.float64, device="cuda")[:, None] * BASE ** (-torch.arange(0, turned, 2, dtype=torch.float64, device="cuda") / max(turned, 1))
    return angle.cos().float(), angle.sin().float()


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, B, H, Hk, d = DTYPES[c["dtype"]], c["B"], c["heads"], c["kv"], c["d"]
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    if c["op"] in ("qk", "qk_bwd"):
        N = c["N"]
        X = (randn(B, N, H + 2 * Hk, d) * torch.exp(0.5 * randn(H + 2 * Hk, d))).to(dt)     # the projection's output, channels of different sizes
        s = dict(c, Q=X[:, :, :H], K=X[:, :, H:H + Hk], q_gamma=None, k_gamma=None, cos=None, sin=None, positions=None)
        if c["norm"]:
            s["q_gamma"], s["k_gamma"] = 1 + 0.1 * randn(d), 1 + 0.1 * randn(d)
        if c["turned"]:
            s["cos"], s["sin"] = _table(N + c["far"], c["turned"])
            if c["far"]:
                start = torch.randint(0, c["far"] + 1, (B, 1), generator=g, device="cuda")
                s["positions"] = (start + torch.arange(N, device="cuda")).to(torch.int32)
        if c["op"] == "qk_bwd":
            s["dQ"], s["dK"] = randn(B, N, H, d).to(dt), randn(B, N, Hk, d).to(dt)
        return s
    Nq, Nk = c["Nq"], c["Nk"]
    if c["where"] == "packed":
        X = randn(B, Nq, H + 2 * Hk, d).to(dt)
        Q, K, V = X[:, :, :H], X[:, :, H:H + Hk], X[:, :, H + Hk:]
    else:
        Q = randn(B, Nq, H, d).to(dt)
        cache = (lambda: randn(B, Hk, Nk, d).to(dt).transpose(1, 2)) if c["where"] == "cache" else (lambda: randn(B, Nk, Hk, d).to(dt))
        K, V = cache(), cache()
    s = dict(c, Q=Q, K=K, V=V, q_lens=None, k_lens=None)
    order = torch.randperm(B, generator=g, device="cuda")
    lengths = lambda n: torch.tensor(_lengths(n, B), dtype=torch.int32, device="cuda")[order]
    if c["q_ragged"]:
        s["q_lens"] = lengths(Nq)
    if c["k_ragged"]:
        s["k_lens"] = lengths(Nk)
    if c["op"] == "att_bwd":
        O, s["lse"] = _attention(s)
        s["O"], s["dO"] = O.to(dt), randn(B, Nq, H, d).to(dt)
    return s


# -- plain forms -------------------------------------------------------------------------------------------------

def _turn(x, s, back):
    """The first `turned` channels rotated in pairs, by the angles of each token's position."""
    r = s["turned"]
    if not r:
        return x
    cos, sin = (s[k] if s["positions"] is None else s[k][s["positions"].long()] for k in ("cos", "sin"))
    cos, sin = (t[..., :x.shape[1], None, :] for t in (cos, -sin if back else sin))
    halves = s["pairs"] == "halves"
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if halves else (x[..., 0:r:2], x[..., 1:r:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([a, b], -1) if halves else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _heads_forward(x, gamma, s):
    x = x.float()
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma
    return _turn(x, s, False)


def _heads_backward(x, dy, gamma, s):
    g = _turn(dy.float(), s, True)
    if gamma is None:
        return g, None
    x = x.float()
    inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    u, du = x * inv, g * gamma
    return inv * (du - u * (du * u).mean(-1, keepdim=True)), (g * u).sum((0, 1, 2))


def _by_head(t, kv):
    """[B, N, heads, d] -> [B, kv, heads / kv * N, d] in 32 bits."""
    B, N, h, d = t.shape
    return t.float().transpose(1, 2).reshape(B, kv, h // kv * N, d)


def _by_token(t, N):
    B, kv, rows, d = t.shape
    return t.view(B, kv * (rows // N), N, d).transpose(1, 2)


def _visible(s):
    """[B or 1, 1, 1, Nq, Nk]: which keys each query sees; the last query of a causal sequence sees all of its keys."""
    Nq, Nk = s["Nq"], s["Nk"]
    i, j = torch.arange(Nq, device="cuda")[:, None], torch.arange(Nk, device="cuda")
    nq = Nq if s["q_lens"] is None else s["q_lens"].view(-1, 1, 1)
    nk = Nk if s["k_lens"] is None else s["k_lens"].view(-1, 1, 1)
    see = (i < nq) & (j < nk)
    if s["causal"]:
        see = see & (j <= i + (nk - nq))
    return see.view(-1, 1, 1, Nq, Nk)


def _logits(s):
    q, k = _by_head(s["Q"], s["kv"]), _by_head(s["K"], s["kv"])
    a = (q @ k.transpose(-1, -2)).mul_(s["d"] ** -0.5)
    return a.view(s["B"], s["kv"], s["heads"] // s["kv"], s["Nq"], s["Nk"])


def _attention(s):
    """O [B, Nq, heads, d] and the logarithm of the sum of exponentials [B, heads, Nq]."""
    a = _logits(s).masked_fill_(~_visible(s), -math.inf)
    top = a.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = a.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = p.view(s["B"], s["kv"], -1, s["Nk"]) @ _by_head(s["V"], s["kv"])
    o = o / torch.where(total == 0, 1.0, total).view(s["B"], s["kv"], -1, 1)
    return _by_token(o, s["Nq"]), (top + torch.log(total)).view(s["B"], s["heads"], s["Nq"])


def _attention_gradients(s):
    B, kv, Nq, Nk, scale = s["B"], s["kv"], s["Nq"], s["Nk"], s["d"] ** -0.5
    lse = s["lse"].view(B, kv, -1, Nq, 1)
    p = torch.where(_visible(s), (_logits(s) - lse).exp_(), 0.0).view(B, kv, -1, Nk)
    q, k, v, o, do = (_by_head(s[n], kv) for n in ("Q", "K", "V", "O", "dO"))
    ds = p * ((do @ v.transpose(-1, -2)) - (do * o).sum(-1, keepdim=True))
    dq, dk, dv = ds @ k * scale, ds.transpose(-1, -2) @ q * scale, p.transpose(-1, -2) @ do
    return [_by_token(dq, Nq), _by_token(dk, Nk), _by_token(dv, Nk)]


def run(s):
    dt = DTYPES[s["dtype"]]
    if not own:
        if s["op"] == "qk":
            return [_heads_forward(s[t], s[g], s).to(dt) for t, g in (("Q", "q_gamma"), ("K", "k_gamma"))]
        if s["op"] == "qk_bwd":
            (dq, gq), (dk, gk) = (_heads_backward(s[t], s["d" + t], s[g], s) for t, g in (("Q", "q_gamma"), ("K", "k_gamma")))
            return [dq.to(dt), dk.to(dt)] + ([gq, gk] if s["norm"] else [])
        if s["op"] == "att":
            o, lse = _attention(s)
            return [o.to(dt), lse] if s["lse"] else [o.to(dt)]
        return [t.to(dt) for t in _attention_gradients(s)]
    import paper_2303_08810_amd as bra
    if s["op"] in ("qk", "qk_bwd"):
        rule = dict(cos=s["cos"], sin=s["sin"], positions=s["positions"], pairs=s["pairs"], eps=EPS)
        if s["op"] == "qk":
            return list(bra.bra_qk_norm_forward(s["Q"], s["K"], s["q_gamma"], s["k_gamma"], **rule))
        return list(bra.bra_qk_norm_backward(s["Q"], s["K"], s["dQ"], s["dK"], s["q_gamma"], s["k_gamma"], **rule))
    rule = dict(causal=s["causal"], q_lens=s["q_lens"], k_lens=s["k_lens"])
    if s["op"] == "att":
        out = bra.bra_attention_forward(s["Q"], s["K"], s["V"], want_lse=s["lse"], **rule)
        return list(out) if s["lse"] else [out]
    return list(bra.bra_attention_backward(s["Q"], s["K"], s["V"], s["O"], s["lse"], s["dO"], **rule))


def work(c):
    b, B, H, Hk, d = BYTES[c["dtype"]], c["B"], c["heads"], c["kv"], c["d"]
    if c["op"] in ("qk", "qk_bwd"):
        n, back = B * c["N"] * (H + Hk) * d, c["op"] == "qk_bwd"
        rows = B * c["N"] if c["far"] else c["N"]
        reads = 2 if back and c["norm"] else 1
        return {"bytes": (reads + 1) * n * b + 4 * rows * c["turned"], "flops": (18.0 if back else 10.0) * n}
    nq = _lengths(c["Nq"], B) if c["q_ragged"] else [c["Nq"]] * B
    nk = _lengths(c["Nk"], B) if c["k_ragged"] else [c["Nk"]] * B
    if c["causal"]:
        # the first max(0, nq - nk) queries see nothing, the others one key more each
        seen = lambda m, n: m * n - m * (m - 1) // 2 if m <= n else n * (n + 1) // 2
        pairs = sum(seen(m, n) for m, n in zip(nq, nk))
    else:
        pairs = sum(m * n for m, n in zip(nq, nk))
    q, k, whole = sum(nq) * H * d * b, sum(nk) * Hk * d * b, B * c["Nq"] * H
    if c["op"] == "att":
        return {"bytes": q + whole * d * b + 2 * k + (4 * whole if c["lse"] else 0), "flops": 4.0 * d * H * pairs}
    return {"bytes": 3 * q + whole * d * b + 2 * k + 2 * B * c["Nk"] * Hk * d * b + 4 * sum(nq) * H, "flops": 10.0 * d * H * pairs}


# -- in 64 bits, from the definitions ----------------------------------------------------------------------------

def _exact_heads(c, s, x, gamma):
    """Norm and rotation as products of complex numbers."""
    if gamma is not None:
        x = x * (x.square().sum(-1, keepdim=True) / c["d"] + EPS).rsqrt() * gamma
    r = c["turned"]
    if not r:
        return x
    unit = torch.complex(s["cos"].double(), s["sin"].double())
    at = torch.arange(c["N"], device="cuda").expand(c["B"], -1) if s["positions"] is None else s["positions"].long()
    unit = unit[at].unsqueeze(2)
    if c["pairs"] == "halves":
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * unit
        return torch.cat([z.real, z.imag, x[..., r:]], -1)
    z = torch.view_as_complex(x[..., :r].reshape(*x.shape[:-1], r // 2, 2)) * unit
    return torch.cat([torch.view_as_real(z).reshape(*x.shape[:-1], r), x[..., r:]], -1)


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] in ("qk", "qk_bwd"):
        live = {k: s[k].double().requires_grad_() for k in ("Q", "K", "q_gamma", "k_gamma") if s[k] is not None}
        q = _exact_heads(c, s, live["Q"], live.get("q_gamma"))
        k = _exact_heads(c, s, live["K"], live.get("k_gamma"))
        if c["op"] == "qk":
            return [q.detach(), k.detach()]
        return list(torch.autograd.grad((q * s["dQ"].double()).sum() + (k * s["dK"].double()).sum(), list(live.values())))
    B, H, G, Nq, Nk, scale = c["B"], c["heads"], c["heads"] // c["kv"], c["Nq"], c["Nk"], 1 / math.sqrt(c["d"])
    back = c["op"] == "att_bwd"
    Q, K, V = (s[n].double() for n in ("Q", "K", "V"))
    out = [torch.zeros_like(t, memory_format=torch.contiguous_format) for t in ((Q, K, V) if back else (Q,))]
    lse = torch.full((B, H, Nq), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        m = Nq if s["q_lens"] is None else int(s["q_lens"][b])
        n = Nk if s["k_lens"] is None else int(s["k_lens"][b])
        hidden = torch.ones(m, n, dtype=torch.bool, device="cuda").triu(n - m + 1) if c["causal"] else None
        for h in range(H):
            q, k, v = Q[b, :m, h], K[b, :n, h // G], V[b, :n, h // G]
            a = torch.mm(q, k.t()) * scale
            if hidden is not None:
                a.masked_fill_(hidden, -math.inf)
            if not back:
                lse[b, h, :m] = torch.logsumexp(a, 1)
                out[0][b, :m, h] = torch.softmax(a, 1).nan_to_num_(0.0).mm(v)
                continue
            p = torch.exp(a - s["lse"][b, h, :m].double()[:, None])
            if hidden is not None:
                p.masked_fill_(hidden, 0.0)
            do, o = s["dO"][b, :m, h].double(), s["O"][b, :m, h].double()
            out[2][b, :n, h // G] += p.t().mm(do)
            e = (do.mm(v.t()) - (do * o).sum(1)[:, None]).mul_(p).mul_(scale)
            out[0][b, :m, h] = e.mm(k)
            out[1][b, :n, h // G] += e.t().mm(q)
    return out if back or not c["lse"] else [out[0], lse]
