"""The norms around a residual sum and their gradients in 64 bits, with bounds on what float32 arithmetic may be off.

U = 2^-24.  A row's sum goes through at most 16 additions in a thread and 9 levels of lanes and wavefronts, so that it is off by less
than 32 U of the sum of the magnitudes; sums over rows through at most as many additions as there are rows.  Centred values are off by the
mean's error e, the deviation by the same and 20 U of itself, hence a normalised value by e / sigma (1 + |u|) + 24 U |u|."""
import torch

U = 2.0 ** -24
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def unit64(x, kind, eps):
    """Normalised rows, one over their deviation, the error of both (the second relative)."""
    mean = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    e = 34 * U * x.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    d = x - mean
    inv = 1 / ((d * d).mean(-1, keepdim=True) + eps).sqrt()
    u = d * inv
    return u, inv, e * inv * (1 + u.abs()) + 24 * U * u.abs(), e * inv + 24 * U


def expand_gate(gate, X):
    """The gate's rows as X's, [rows, C]."""
    C = X.shape[-1]
    rows, g = X.numel() // C, gate.double().reshape(-1, C)
    return g.repeat_interleave(rows // max(1, g.shape[0]), 0)


def flat(t):
    return t.double().reshape(-1, t.shape[-1])


def forward64(X, Y, P, kind, eps):
    """R and its error before rounding, and N's."""
    x = flat(X)
    if Y is None:
        r, er = x, torch.zeros_like(x)
    else:
        z, ez = flat(Y), torch.zeros_like(x)
        if P.get("post_gamma") is not None:
            u, _, eu, _ = unit64(z, kind, eps)
            pg, pb = P["post_gamma"].double(), P["post_beta"].double() if P.get("post_beta") is not None else 0.0
            z = u * pg + pb
            ez = eu * pg.abs() + 3 * U * (u * pg).abs() + U * z.abs()
        k = torch.ones_like(x)
        if P.get("scale") is not None:
            k = k * P["scale"].double()
        if P.get("gate") is not None:
            k = k * expand_gate(P["gate"], X)
        r = x + k * z
        er = k.abs() * ez + 3 * U * (k * z).abs() + U * r.abs()
    if P.get("gamma") is None:
        return r, er, None, None
    u, inv, eu, rel = unit64(r, kind, eps)
    gamma, beta = P["gamma"].double(), P["beta"].double() if P.get("beta") is not None else 0.0
    n = u * gamma + beta
    # the sum's own error moves the row by itself and by its mean and deviation
    moved = (er + er.mean(-1, keepdim=True)) * inv + u.abs() * (er * u.abs()).mean(-1, keepdim=True) * inv
    return r, er, n, (eu + moved) * gamma.abs() + 3 * U * (u * gamma).abs() + U * n.abs()


def check(got, ref, bound, unit, name):
    got = got.double().reshape(ref.shape)
    assert torch.isfinite(got).all(), name
    if not got.numel():
        return
    worst = float(((got - ref).abs() / (1.01 * bound + unit * (ref.abs() + bound) + 1e-37)).max())
    assert worst <= 1.0, (name, worst)


def check_forward(R, N, X, Y, P, kind, eps):
    r, er, n, en = forward64(X, Y, P, kind, eps)
    if R is not None:
        check(R, r, er, UNIT[X.dtype], "R")
    if N is not None:
        check(N, n, en, UNIT[X.dtype], "N")


def check_backward(grads, R, Y, P, dN, dR, kind, eps):
    x, unit = flat(R), UNIT[R.dtype]
    rows = x.shape[0]
    want = {"dX"}
    D, eD = (flat(dR), torch.zeros_like(x)) if dR is not None else (torch.zeros_like(x), torch.zeros_like(x))
    over_rows = lambda t, e: (t.sum(0), e.sum(0) + (rows + 80) * U * t.abs().sum(0))
    if dN is not None:
        u, inv, eu, rel = unit64(x, kind, eps)
        dn, gamma = flat(dN), P["gamma"].double()
        g = dn * gamma
        m1 = g.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(inv)
        m2 = (g * u).mean(-1, keepdim=True)
        e1, e2 = 36 * U * g.abs().mean(-1, keepdim=True), 36 * U * (g * u).abs().mean(-1, keepdim=True) + (g.abs() * eu).mean(-1, keepdim=True)
        b = inv * (g - m1 - u * m2)
        eD = inv * (3 * U * g.abs() + e1 + u.abs() * e2 + eu * m2.abs() + 3 * U * (m1.abs() + (u * m2).abs())) + rel * b.abs() + 2 * U * (b.abs() + D.abs())
        D = D + b
        want |= {"dgamma", "dbeta"}
        check(grads["dgamma"], *over_rows(dn * u, dn.abs() * eu), U, "dgamma")
        check(grads["dbeta"], *over_rows(dn, torch.zeros_like(dn)), U, "dbeta")
    check(grads["dX"], D, eD, unit, "dX")
    if Y is not None:
        want |= {"dY"}
        y, post = flat(Y), P.get("post_gamma") is not None
        one = torch.ones_like(x)
        scale = P["scale"].double() if P.get("scale") is not None else torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
        gate = expand_gate(P["gate"], R) if P.get("gate") is not None else one
        if post:
            yu, yinv, eyu, yrel = unit64(y, kind, eps)
            pg, pb = P["post_gamma"].double(), P["post_beta"].double() if P.get("post_beta") is not None else torch.zeros_like(scale)
        else:
            yu, eyu, pg, pb = y, torch.zeros_like(y), torch.ones_like(scale), torch.zeros_like(scale)
        Z, eZ = yu * pg + pb, eyu * pg.abs() + 2 * U * ((yu * pg).abs() + pb.abs())
        terms, eT = D * Z, eD * Z.abs() + (D.abs() + eD) * eZ + 4 * U * D.abs() * ((yu * pg).abs() + pb.abs())
        mag = D.abs() * ((yu * pg).abs() + pb.abs())
        if P.get("scale") is not None:
            want.add("dscale")
            t = gate * terms
            check(grads["dscale"], t.sum(0), (gate.abs() * eT).sum(0) + (rows + 90) * U * (gate.abs() * mag).sum(0), U, "dscale")
        if P.get("gate") is not None:
            want.add("dgate")
            G = P["gate"].numel() // x.shape[1]
            per = rows // G
            fold = lambda t: t.view(G, per, -1).sum(1)
            check(grads["dgate"], fold(scale * terms), scale.abs() * (fold(eT) + (per + 90) * U * fold(mag)), unit, "dgate")
        dZ, edZ = D * scale * gate, (eD + 4 * U * D.abs()) * (scale * gate).abs()
        if post:
            want |= {"dpost_gamma", "dpost_beta"}
            check(grads["dpost_gamma"], *over_rows(dZ * yu, edZ * yu.abs() + dZ.abs() * eyu), U, "dpost_gamma")
            check(grads["dpost_beta"], *over_rows(dZ, edZ), U, "dpost_beta")
            t, et = dZ * pg, edZ * pg.abs() + 2 * U * (dZ * pg).abs()
            m1 = t.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(yinv)
            m2 = (t * yu).mean(-1, keepdim=True)
            e1 = et.mean(-1, keepdim=True) + 36 * U * t.abs().mean(-1, keepdim=True)
            e2 = (et * yu.abs() + t.abs() * eyu).mean(-1, keepdim=True) + 36 * U * (t * yu).abs().mean(-1, keepdim=True)
            b = yinv * (t - m1 - yu * m2)
            dZ = b
            edZ = yinv * (et + e1 + yu.abs() * e2 + eyu * m2.abs() + 3 * U * (t.abs() + m1.abs() + (yu * m2).abs())) + yrel * b.abs()
        check(grads["dY"], dZ, edZ, unit, "dY")
    assert set(grads) == want, (set(grads), want)
