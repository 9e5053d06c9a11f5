"""The dense block in front of the layer and the losses against short lists, from their definitions, in 64 bits on the CPU."""
import math

import torch

U = 2.0 ** -24   # a rounding to float32, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def act(a, kind):
    if kind == 0:
        return a * torch.sigmoid(a)
    return a * 0.5 * torch.special.erfc(-a / math.sqrt(2.0))


def slope(a, kind):
    if kind == 0:
        p = torch.sigmoid(a)
        return p + a * p * torch.sigmoid(-a)
    return 0.5 * torch.special.erfc(-a / math.sqrt(2.0)) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)


def gated(e, Vg, Vu, kind):
    """gate, up, x and the bounds of their errors before the last rounding: a sum of w products in any order, twice w roundings at most; act' is below 1.13,
    and act itself (an exponential or an error function, 4 more operations) off by 8 roundings of |gate|."""
    e, Vg, Vu = e.double().cpu(), Vg.double().cpu(), Vu.double().cpu()
    a, u = e @ Vg.t(), e @ Vu.t()
    n = 2 * e.shape[1] + 8
    da, du = n * U * (e.abs() @ Vg.abs().t()), n * U * (e.abs() @ Vu.abs().t())
    x = act(a, kind) * u
    dv = 1.13 * da + 8 * U * a.abs()
    dx = dv * (u.abs() + du) + act(a, kind).abs() * du + 2 * U * x.abs()
    return (a, da), (u, du), (x, dx)


def gated_backward(grad_x, e, Vg, Vu, gate, up, kind):
    """grad_e, grad_V_gate, grad_V_up with the bounds of their elements' errors and of their norms' (relative).  A factor of G is off by 8 roundings of
    1 + |gate| of it; a sum of K products by 2 K roundings at most, by a random walk of them, U * sqrt(K / 6), as a norm."""
    g, e, Vg, Vu, a, u = (t.double().cpu() for t in (grad_x, e, Vg, Vu, gate, up))
    ga, gu = g * u * slope(a, kind), g * act(a, kind)
    dga, dgu = 10 * U * (g * u).abs() * (1 + a.abs()), 10 * U * g.abs() * (1 + a.abs())
    b, d = g.shape

    def bound(G, dG, M, K):
        return (2 * K + 8) * U * (G.abs() @ M.abs()) + dG @ M.abs()

    ge = ga @ Vg + gu @ Vu
    out = [(ge, bound(ga, dga, Vg, 2 * d) + bound(gu, dgu, Vu, 2 * d), U * (16 + math.sqrt(2 * d)))]
    for G, dG in ((ga, dga), (gu, dgu)):
        out.append((G.t() @ e, bound(G.t(), dG.t(), e, b), U * (16 + math.sqrt(b))))
    return out


def codes(rows):
    """8-bit codes and scales, to the bit: both quotients are rounded to float32."""
    v = rows.float().cpu()
    top = v.abs().amax(1)
    fine = torch.isfinite(v).all(1)
    scale = torch.clamp((top.double() / 127).float(), min=2.0 ** -126)
    q = torch.round((v.double() / scale.double()[:, None]).float()).clamp(-127, 127)
    q = torch.where(fine[:, None], q, torch.zeros(()))
    return q.to(torch.int8), torch.where(fine, scale, torch.full((), math.nan))


def entries(z, lab, logit=None):
    """Which entries of a row count."""
    m = z.numel()
    return [e for e in range(len(lab)) if 0 <= int(lab[e]) < m and float(z[int(lab[e])]) != -math.inf and (logit is None or float(logit[e]) != -math.inf)]


def distill(out, off, lab, logit, T, scale):
    out, logit = out.double().cpu(), logit.double().cpu()
    off, lab = off.tolist(), lab.cpu()
    g, loss = torch.zeros_like(out), 0.0
    for i in range(out.shape[0]):
        l, t = lab[off[i]:off[i + 1]], logit[off[i]:off[i + 1]]
        counts = entries(out[i], l, t)
        if not counts:
            continue
        at, lp = l[counts].long(), torch.log_softmax(t[counts] / T, 0)
        lq = torch.log_softmax(out[i] / T, 0)
        loss += float((torch.exp(lp) * (lp - lq[at])).sum()) * scale * T * T
        g[i] = torch.exp(lq).index_add(0, at, -torch.exp(lp)) * scale * T
    return g, loss


def policy(out, off, lab, old, ref, adv, low, high, beta, scale):
    out = out.double().cpu()
    off, lab, old, adv = off.tolist(), lab.cpu(), old.double().cpu(), adv.double().cpu()
    ref = ref.double().cpu() if ref is not None else torch.zeros_like(old)
    g, loss, logp = torch.zeros_like(out), 0.0, torch.full_like(old, -math.inf)
    for i in range(out.shape[0]):
        counts = [off[i] + e for e in entries(out[i], lab[off[i]:off[i + 1]])]
        if not counts:
            continue
        z = out[i].clone().requires_grad_()
        lp = torch.log_softmax(z, 0)[lab[counts].long()]
        r, u = torch.exp(lp - old[counts]), ref[counts] - lp
        free, held = r * adv[counts], r.clamp(1 - low, 1 + high) * adv[counts]
        row = torch.where(free <= held, -free, -held.detach()).sum()
        if beta:
            row = row + beta * (torch.exp(u) - u - 1).sum()
        row.backward()
        loss += float(row.detach()) * scale
        g[i] = z.grad * scale
        logp[counts] = lp.detach()
    return g, loss, logp
