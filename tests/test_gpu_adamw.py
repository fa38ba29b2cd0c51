"""GPU tests of the AdamW step: bit for bit against the formula's float32 operations one by one on the CPU (IEEE, no contraction),
against 64 bits, and the 8-bit states' codes against their definition."""
import math

import numpy as np
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
SIZES = [1, 7, 31, 32, 33, 2048, 2049, 64 * 192, 5000, 2, 64, 0, 100000]
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.98, eps=1e-8)


def f32(v):
    return torch.tensor(v, dtype=F32).item()


def power_of_two(e):
    """2^e as torch.ldexp and the kernel have it on the GPU, where powf is a unit off for some exponents (2^-109, 2^17, ..): never more."""
    p = torch.ldexp(torch.ones(e.shape, device="cuda"), e.cuda()).cpu()
    assert ((p.double() / torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e) - 1).abs() <= 2.0 ** -23).all()
    return p


def encode(x, root):
    """As documented: the smallest power of two with which the largest value of 32 is at most 448."""
    x = x.view(-1, 32)
    m, e = torch.frexp(x.abs().amax(1, keepdim=True))
    e = torch.where(m == 0, -126, torch.clamp(e - 9 + (m > 0.875).int(), min=-126))
    q = x * power_of_two(-e)
    if root:
        q = torch.where((q > 0) & (q < 2.0 ** -9), 2.0 ** -9, q)
    return q.to(torch.float8_e4m3fn).view(-1), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu).view(-1)


def decode(codes, scales):
    return (codes.float().view(-1, 32) * power_of_two(scales.view(torch.uint8).int()[:, None] - 127)).view(-1)


def sqrt(v):
    """Correctly rounded: torch's CPU kernel goes through a vector library that is off by a unit on some processors (inputs of
    test_steps_bit_for_bit, tensor 3, element 20: the IEEE root gives 1015969498 as the GPU does, that library's 1015969499)."""
    return torch.from_numpy(np.sqrt(v.numpy()))


def places(params):
    at = 0
    for p in params:
        yield at, p.numel()
        at += (p.numel() + 31) // 32 * 32


def step_cpu(params, grads, state, t, decay, lr, beta1, beta2, eps, grad_scale=None):
    """New parameters (unrounded) and states, float32 operation by operation."""
    bits8 = "exp_avg_root" in state
    M = decode(state["exp_avg"], state["exp_avg_scale"]) if bits8 else state["exp_avg"].clone()
    V = decode(state["exp_avg_root"], state["exp_avg_root_scale"]) if bits8 else state["exp_avg_sq"].clone()
    V, root_all, out = (V * V if bits8 else V), torch.zeros_like(V), []
    away, bias = f32(lr / (1 - beta1 ** t)), f32(1 / math.sqrt(1 - beta2 ** t))
    for (at, n), p, g, wd in zip(places(params), params, grads, decay):
        if g is None or n == 0:
            root_all[at:at + n] = sqrt(V[at:at + n])
            out.append(p.float())
            continue
        p, g, m, v = p.float().flatten(), g.float().flatten(), M[at:at + n], V[at:at + n]
        if grad_scale is not None:
            g = g * grad_scale
        m = f32(beta1) * m + f32(1 - beta1) * g
        v = f32(beta2) * v + f32(1 - beta2) * (g * g)
        root = sqrt(v)
        p = p * f32(1 - lr * f32(wd)) - away * (m / (root * bias + f32(eps)))
        M[at:at + n], V[at:at + n], root_all[at:at + n] = m, v, root
        out.append(p)
    if not bits8:
        return out, {"exp_avg": M, "exp_avg_sq": V}
    new = dict(zip(("exp_avg", "exp_avg_scale"), encode(M, False)))
    new.update(zip(("exp_avg_root", "exp_avg_root_scale"), encode(root_all, True)))
    return out, new


def raw(t):
    return t.cpu().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def tensors(dtype, grad, seed, sizes=SIZES):
    g = torch.Generator().manual_seed(seed)
    r = lambda n: torch.randn(n, generator=g)
    params = [(0.05 * r(n)).to(dtype) for n in sizes]
    steps = [[(1e-3 * r(n) * torch.exp(2 * r(n))).to(grad) for n in sizes] for _ in range(4)]
    return params, steps


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
def test_steps_bit_for_bit(bits, dtype, grad):
    params, steps = tensors(dtype, grad, 7)
    decay = [0.05 * (i % 3) for i in range(len(params))]
    dev = [p.cuda() for p in params]
    copies = [torch.empty_like(p, dtype=BF16) if i % 2 else None for i, p in enumerate(dev)] if dtype == F32 else None
    state = bra.adamw_state(dev, bits)
    cpu_state = {k: v.cpu() for k, v in state.items()}
    for t, grads in enumerate(steps, 1):
        if t == 3:
            grads = [None if i == 4 else g for i, g in enumerate(grads)]        # left alone once
        print(f"adamw bits {bits} {dtype} {grad} step {t}", flush=True)
        before = state["exp_avg"].clone()
        bra.bra_adamw_step(dev, [None if g is None else g.cuda() for g in grads], state, step=t, weight_decay=decay, copies=copies, **HYPER)
        out, new = step_cpu(params, grads, cpu_state, t, decay, **HYPER)
        for i, ((at, n), p, d, o) in enumerate(zip(places(params), params, dev, out)):
            assert torch.equal(raw(d), raw(o.to(dtype))), i
            if grads[i] is None:
                assert torch.equal(raw(before[at:at + n]), raw(state["exp_avg"][at:at + n]))
            elif copies and copies[i] is not None:
                assert torch.equal(raw(copies[i]), raw(o.to(BF16))), i
        params = [o.to(dtype) for o in out]
        for k in new:
            if grads[4] is not None or bits == 32:
                assert torch.equal(raw(state[k]), raw(new[k])), k
        cpu_state = {k: v.cpu() for k, v in state.items()}


def test_against_64_bits():
    """One step: m, v off by three roundings, the parameter by its own, the update's and what they carry."""
    params, steps = tensors(F32, F32, 11)
    dev, state = [p.cuda() for p in params], None
    state = bra.adamw_state(dev)
    bra.bra_adamw_step(dev, [g.cuda() for g in steps[0]], state, step=1, weight_decay=0.1, **HYPER)
    u = 2.0 ** -24
    for (at, n), p, g, d in zip(places(params), params, steps[0], dev):
        p, g = p.double(), g.double()
        m, v = 0.1 * g, 0.02 * g * g
        upd = HYPER["lr"] / 0.1 * m / (v.sqrt() / math.sqrt(0.02) + HYPER["eps"])
        new = p * (1 - HYPER["lr"] * 0.1) - upd
        assert ((state["exp_avg"][at:at + n].cpu().double() - m).abs() <= 4 * u * m.abs() + 1e-44).all()
        assert ((state["exp_avg_sq"][at:at + n].cpu().double() - v).abs() <= 6 * u * v + 1e-44).all()
        assert ((d.cpu().double() - new).abs() <= 4 * u * p.abs() + 24 * u * upd.abs()).all()


def test_roots_of_8_bits_do_not_vanish():
    p = [torch.zeros(64, device="cuda")]
    state = bra.adamw_state(p, 8)
    g = torch.full((64,), 1e-9, device="cuda")
    g[0] = g[40] = 1e3
    bra.bra_adamw_step(p, [g], state, step=1, weight_decay=0.0, **HYPER)
    assert (state["exp_avg_root"].view(torch.uint8) > 0).all()
    before = p[0].clone()
    bra.bra_adamw_step(p, [torch.zeros_like(g)], state, step=2, weight_decay=0.0, **HYPER)
    assert float((p[0] - before).abs().max()) < 2 * HYPER["lr"]


def test_values_that_are_not_finite_stay_where_they_are():
    for bits in (32, 8):
        p = [torch.ones(96, device="cuda")]
        g = torch.ones(96, device="cuda")
        g[5], g[40] = float("nan"), float("inf")
        state = bra.adamw_state(p, bits)
        bra.bra_adamw_step(p, [g], state, step=1, **HYPER)
        bad = ~torch.isfinite(p[0]).cpu()
        assert bad.nonzero().flatten().tolist() == [5, 40], bits
        m = state["exp_avg"].float().cpu()
        assert torch.isfinite(m[64:]).all() and torch.isnan(m[5])


def test_step_on_the_device_and_scale():
    params, steps = tensors(F32, F32, 13)
    a, b = [p.cuda() for p in params], [p.cuda() for p in params]
    sa, sb = bra.adamw_state(a), bra.adamw_state(b)
    t, scale = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0.25], device="cuda")
    for i, grads in enumerate(steps, 1):
        t += 1
        bra.bra_adamw_step(a, [g.cuda() for g in grads], sa, step=t, grad_scale=scale, **HYPER)
        bra.bra_adamw_step(b, [0.25 * g.cuda() for g in grads], sb, step=i, **HYPER)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and all(torch.equal(sa[k], sb[k]) for k in sa)


def test_more_tensors_than_a_launch_takes_and_views():
    sizes = [1 + 37 * i % 300 for i in range(200)]
    total = sum(sizes)
    for bits in (32, 8):
        params, steps = tensors(F32, F32, 17, sizes)
        flat, gflat = torch.cat(params).cuda(), torch.cat(steps[0]).cuda()       # views at every alignment
        dev, grads = list(flat.split(sizes)), list(gflat.split(sizes))
        state = bra.adamw_state(dev, bits)
        cpu_state = {k: v.cpu() for k, v in state.items()}
        bra.bra_adamw_step(dev, grads, state, step=1, weight_decay=0.01, **HYPER)
        out, new = step_cpu(params, steps[0], cpu_state, 1, [0.01] * 200, **HYPER)
        assert torch.equal(raw(flat), raw(torch.cat(out))) and flat.numel() == total
        assert all(torch.equal(raw(state[k]), raw(new[k])) for k in new)


def test_captured_steps():
    params, steps = tensors(F32, F32, 19)
    a, b = [p.cuda() for p in params], [p.cuda() for p in params]
    sa, sb = bra.adamw_state(a), bra.adamw_state(b)
    t, grads = torch.zeros(1, dtype=torch.int32, device="cuda"), [torch.zeros_like(p) for p in a]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        t += 1
        bra.bra_adamw_step(a, grads, sa, step=t, **HYPER)
    for i, new in enumerate(steps, 1):
        for g, n in zip(grads, new):
            g.copy_(n)
        graph.replay()
        bra.bra_adamw_step(b, [n.cuda() for n in new], sb, step=i, **HYPER)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, b)), i
