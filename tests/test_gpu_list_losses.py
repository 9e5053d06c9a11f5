"""Distillation and the policy loss against float64: rows without entries, masked labels, the same label twice, odd sizes, in place, graphs."""
import math

import pytest
import torch

import dense_reference as R
from test_gpu_gated import guarded, untouched, usl

pytestmark = pytest.mark.gpu


def lists(b, m, lengths, seed):
    gen = torch.Generator().manual_seed(seed)
    off = torch.tensor([0] + list(lengths), dtype=torch.int64).cumsum(0)
    lab = torch.cat([torch.randperm(m, generator=gen)[:n] if n <= m else torch.randint(0, m, (n,), generator=gen) for n in lengths]
                    + [torch.zeros(0, dtype=torch.int64)]).to(torch.int32)
    return off, lab, gen


def layer(m, b, stream=None):
    return usl().Layer(m, 4, 1, b, "f32", stream or torch.cuda.current_stream().cuda_stream)


def tolerance(out, T, want_g, entry_sum):
    """q is off by the roundings of its exponent (2 of |z - top| / T), of the exponential and of the sum's lanes and joins (below 32): all relative; the entries by 4
    roundings of theirs, and the result by one."""
    z = out.double().cpu()
    fine = torch.where(torch.isfinite(z), z, torch.zeros(()).double())   # (rows of others list nothing: no tolerance there)
    span = (fine.amax(1, keepdim=True) - fine.amin(1, keepdim=True)) / T
    return (2 * span + 40) * R.U * (want_g.abs() + entry_sum) + 2 * R.U * want_g.abs() + 1e-38


def distill_case(out, off, lab, logit, T, scale, in_place=False, L=None):
    b, m = out.shape
    own = L or layer(m, b)
    loss, ls = guarded(1)
    g, gs = guarded(b, m, shift=1)
    src = out.cuda()
    if in_place:
        g.copy_(src)
        src = g
    own.distill_loss_grad(src, off.cuda(), lab.cuda(), logit.float().cuda(), T, scale, g, loss, b)
    want, want_loss = R.distill(out, off, lab, logit.float(), T, scale)
    p = torch.zeros_like(want)   # p of the entries
    for i in range(b):
        l, t = lab[off[i]:off[i + 1]], logit[off[i]:off[i + 1]].double()
        c = R.entries(out[i], l, t)
        if c:
            p[i].index_add_(0, l[c].long(), torch.softmax(t[c] / T, 0))
    err = (g.double().cpu() - want).abs()
    worst = float((err / tolerance(out, T, want, scale * T * p)).max())
    assert worst <= 1.0, "g: worst error over its bound %.3g" % worst
    rows = int((off.diff() > 0).sum())
    assert abs(float(loss) - want_loss) <= scale * T * T * rows * 40 * R.U * (1 + float(out[out > -math.inf].abs().max()) / T) + R.U * abs(want_loss), (float(loss), want_loss)
    assert untouched(g, gs) and untouched(loss, ls)
    alone = torch.full((1,), math.nan, device="cuda")
    if not in_place:
        own.distill_loss_grad(src, off.cuda(), lab.cuda(), logit.float().cuda(), T, scale, None, alone, b)
        assert torch.equal(alone, loss)
    if L is None:
        own.close()
    return g


SIZES = [(1, 1, [1]), (1, 5, [3]), (3, 64, [0, 10, 1]), (4, 1000, [5, 0, 0, 40]), (2, 4095, [3, 4]), (2, 4096, [3, 4]), (2, 4097, [100, 4]), (5, 8191, [0, 0, 7, 0, 1]),
         (3, 8193, [1, 300, 2]), (2, 20001, [1000, 64]), (1, 70001, [32]), (70, 3001, [i % 7 for i in range(70)]), (2, 33000, [2000, 1]), (3, 65536, [70, 0, 1500]),
         (2, 65537, [9, 1100]), (300, 1024, [i % 5 for i in range(300)]), (2, 32768, [4, 5000]), (2, 1025, [1025, 3])]


@pytest.mark.parametrize("b,m,lengths", SIZES)
def test_distill(b, m, lengths):
    off, lab, gen = lists(b, m, lengths, m)
    out = torch.randn(b, m, generator=gen) * 3
    logit = torch.randn(lab.numel(), generator=gen) * 4
    for T, scale in ((1.0, 1.0), (2.0, 0.37), (0.5, 1.0 / b)):
        distill_case(out, off, lab, logit, T, scale)
    distill_case(out, off, lab, logit, 3.0, 1.0, in_place=True)


def hard_lists(m):
    """Labels twice and often, outside, masked; logits of -infinity; rows where nothing counts, a row without scores."""
    gen = torch.Generator().manual_seed(5)
    out = torch.randn(9, m, generator=gen) * 2
    rows = [[3, 3, 3, 8999, 3, 4096, 4095], [-1, m, 2 ** 31 - 1, -2 ** 31, 7], [10, 11], [12, 12, 13], [], [-5, m], [100, 200], [5] * 700 + [6, 5], [20, 20]]
    out[2, 10], out[2, 11] = -math.inf, -math.inf           # nothing counts
    out[3, 12], out[3, 100:4500] = -math.inf, -math.inf     # one entry does
    out[5, :] = math.nan                                    # not looked at
    out[6, :] = -math.inf                                   # no label left
    out[8, :4096] = -math.inf                               # a whole segment masked, with the entries in it ...
    out[8, 20] = -1000.0                                    # ... but for one label far below the others
    off = torch.tensor([0] + [len(r) for r in rows]).cumsum(0)
    lab = torch.tensor([l for r in rows for l in r], dtype=torch.int64).to(torch.int32)
    logit = torch.randn(lab.numel(), generator=gen) * 3
    logit[0], logit[4] = -math.inf, -math.inf
    return out, off, lab, logit, gen


@pytest.mark.parametrize("wide", [9000, 65537])
def test_distill_of_hard_lists(wide):
    out, off, lab, logit, _ = hard_lists(wide)
    for in_place in (False, True):
        g = distill_case(out, off, lab, logit, 1.5, 0.5, in_place=in_place)
        assert bool((g[[2, 4, 5, 6]] == 0).all()) and bool((g[1] != 0).any())


def test_temperatures_far_from_one():
    """Logits and scores whose quotients by T leave float32's range, and those that vanish in it: the entries count all the same."""
    off, lab, gen = lists(2, 6000, [3, 2], 3)
    out = torch.randn(2, 6000, generator=gen)
    L = layer(6000, 2)
    for T, size in ((1e-30, 1e12), (1e30, 1.0)):
        logit = torch.randn(5, generator=gen) * size
        g, loss = torch.empty(2, 6000, device="cuda"), torch.empty(1, device="cuda")
        L.distill_loss_grad(out.cuda(), off.cuda(), lab.cuda(), logit.cuda(), T, 1.0 / T if T > 1 else 1e30, g, loss, 2)
        # scale * T = 1: g = q - p, q one-hot or flat, p one-hot or flat
        want = torch.zeros(2, 6000)
        for i in range(2):
            want[i] = torch.softmax(out[i].double() / T, 0).float()
            e = slice(int(off[i]), int(off[i + 1]))
            want[i].index_add_(0, lab[e].long(), -torch.softmax(logit[e].double() / T, 0).float())
        assert torch.allclose(g.cpu(), want, rtol=1e-5, atol=1e-6), (T, float((g.cpu() - want).abs().max()))
    L.close()


def policy_case(out, off, lab, old, ref, adv, low, high, beta, scale, in_place=False, L=None):
    b, m = out.shape
    own = L or layer(m, b)
    n = lab.numel()
    loss, ls = guarded(1)
    g, gs = guarded(b, m, shift=3)
    logp, ps = guarded(max(n, 1))
    src = out.cuda()
    if in_place:
        g.copy_(src)
        src = g
    args = [off.cuda(), lab.cuda(), old.cuda(), ref.cuda() if ref is not None else None, adv.cuda(), low, high, beta, scale]
    own.policy_loss_grad(src, *args, g, logp, loss, b)
    want, want_loss, want_logp = R.policy(out, off, lab, old, ref, adv, low, high, beta, scale)
    # logp is off by the sum's 32 roundings and its own; a slope by as much of what is exponentiated
    d = (logp[:n].double().cpu() - want_logp).abs()
    counts = want_logp > -math.inf
    assert bool((logp[:n].cpu()[~counts] == -math.inf).all())
    if bool(counts.any()):
        assert bool((d[counts] <= 40 * R.U + 2 * R.U * want_logp[counts].abs()).all())
    r = torch.exp(torch.where(counts, want_logp, old.double()) - old.double())
    size = (r * adv.double().abs() + (beta * (1 + torch.exp(ref.double() - torch.where(counts, want_logp, ref.double()))) if ref is not None else 0.0)) * counts
    at = torch.zeros_like(want)
    total = torch.zeros(b, dtype=torch.float64)
    for i in range(b):
        for e in range(int(off[i]), int(off[i + 1])):
            if bool(counts[e]):
                at[i, int(lab[e])] += float(size[e])
                total[i] += float(size[e])
    z = torch.where(counts.any(), out.double(), 0.0)
    live = torch.where(torch.isnan(z), torch.full((), -math.inf).double(), z)
    q = torch.softmax(torch.where((live > -math.inf).any(1, keepdim=True), live, torch.zeros(()).double()), 1)
    span = torch.where(live == -math.inf, torch.zeros(()).double(), live)
    span = span.amax(1, keepdim=True) - span.amin(1, keepdim=True)
    room = scale * (2 * span + 80) * R.U * (at + q * total[:, None]) + 1e-38
    worst = float(((g.double().cpu() - want).abs() / room).max())
    assert worst <= 1.0, "g: worst error over its bound %.3g" % worst
    whole = scale * float((size + adv.double().abs() * (1 + high) * counts).sum())
    assert abs(float(loss) - want_loss) <= 80 * R.U * whole + scale * beta * 40 * R.U * n + R.U * abs(want_loss), (float(loss), want_loss)
    assert untouched(g, gs) and untouched(loss, ls) and untouched(logp, ps)
    if not in_place:
        alone, logp2 = torch.full((1,), math.nan, device="cuda"), torch.full((max(n, 1),), math.nan, device="cuda")
        own.policy_loss_grad(src, *args, None, logp2, alone, b)
        assert torch.equal(alone, loss) and torch.equal(logp2[:n], logp[:n])
        own.policy_loss_grad(src, *args, None, None, alone, b)
        assert torch.equal(alone, loss)
    if L is None:
        own.close()
    return g


def policy_values(out, off, lab, gen):
    n = lab.numel()
    z = out.double()
    at = torch.tensor([float(torch.log_softmax(z[i], 0)[int(lab[e])]) if 0 <= int(lab[e]) < z.shape[1] else -3.0 for i in range(z.shape[0]) for e in range(int(off[i]), int(off[i + 1]))])
    at = torch.where(torch.isfinite(at), at, torch.full((), -3.0))
    return (at + 0.4 * torch.randn(n, generator=gen)).float(), (at + 0.4 * torch.randn(n, generator=gen)).float(), torch.randn(n, generator=gen)


@pytest.mark.parametrize("b,m,lengths", SIZES)
def test_policy(b, m, lengths):
    off, lab, gen = lists(b, m, lengths, m + 1)
    out = torch.randn(b, m, generator=gen) * 3
    old, ref, adv = policy_values(out, off, lab, gen)
    policy_case(out, off, lab, old, ref, adv, 0.2, 0.28, 0.05, 1.0 / lab.numel())
    policy_case(out, off, lab, old, None, adv, 0.2, 0.2, 0.0, 1.0)
    policy_case(out, off, lab, old, ref, adv, 1.0, 0.0, 1.0, 0.25, in_place=True)


@pytest.mark.parametrize("wide", [9000, 65537])
def test_policy_of_hard_lists(wide):
    out, off, lab, _, gen = hard_lists(wide)
    old, ref, adv = policy_values(out, off, lab, gen)
    last = slice(int(off[8]), int(off[9]))
    old[last] = ref[last] = -1000.0   # (of the label far below the others: the ratio stays a number)
    for in_place in (False, True):
        g = policy_case(out, off, lab, old, ref, adv, 0.2, 0.28, 0.1, 0.5, in_place=in_place)
        assert bool((g[[2, 4, 5, 6]] == 0).all())


def test_a_ratio_at_its_bounds():
    """Clipped where the advantage says so, and not on the other side: the four cases, from ratios of 1/2, 1 and 2."""
    m = 10
    out = torch.zeros(1, m)
    lp = -math.log(m)
    old = torch.tensor([lp - math.log(r) for r in (0.5, 1.0, 2.0)] * 2).float()
    adv = torch.tensor([1.0] * 3 + [-1.0] * 3)
    off, lab = torch.tensor([0, 6]), torch.arange(6, dtype=torch.int32)
    L = layer(m, 1)
    g, loss, logp = torch.empty(1, m, device="cuda"), torch.empty(1, device="cuda"), torch.empty(6, device="cuda")
    L.policy_loss_grad(out.cuda(), off.cuda(), lab.cuda(), old.cuda(), None, adv.cuda(), 0.2, 0.2, 0.0, 1.0, g, logp, loss, 1)
    c = torch.tensor([-0.5, -1.0, 0.0, 0.0, 1.0, 2.0])
    want = torch.zeros(m)
    want[:6] = c
    want -= c.sum() / m
    assert torch.allclose(g[0].cpu(), want, rtol=0, atol=1e-5)
    assert abs(float(loss) - (-(0.5 + 1.0 + 1.2) + (0.8 + 1.0 + 2.0))) < 1e-5
    L.close()


def test_nothing_is_listed():
    """Lists without an entry, and a tensor without elements."""
    out = torch.randn(3, 500).cuda()
    off = torch.zeros(4, dtype=torch.int64, device="cuda")
    none_i, none_f = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    L = layer(500, 3)
    g, loss = torch.full((3, 500), math.nan, device="cuda"), torch.full((1,), math.nan, device="cuda")
    L.distill_loss_grad(out, off, none_i, none_f, 1.0, 1.0, g, loss, 3)
    assert bool((g == 0).all()) and float(loss) == 0.0
    g.fill_(math.nan)
    loss.fill_(math.nan)
    L.policy_loss_grad(out, off, none_i, none_f, none_f, none_f, 0.2, 0.2, 0.1, 1.0, g, none_f, loss, 3)
    assert bool((g == 0).all()) and float(loss) == 0.0
    L.close()


@pytest.mark.parametrize("m", [9001, 66000])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_scores_that_are_not_numbers(bad, m):
    """NaN or +infinity anywhere in a row that lists an entry: NaN there, and the other rows as without it."""
    out = torch.randn(3, m)
    off, lab = torch.tensor([0, 2, 4, 6]), torch.tensor([1, 2, 3, 4, 5, 6], dtype=torch.int32)
    logit = torch.randn(6)
    L = layer(m, 3)
    clean, dirty, loss = torch.empty(3, m, device="cuda"), torch.empty(3, m, device="cuda"), torch.empty(1, device="cuda")
    L.distill_loss_grad(out.cuda(), off.cuda(), lab.cuda(), logit.cuda(), 1.0, 1.0, clean, loss, 3)
    out[1, 7000] = bad
    L.distill_loss_grad(out.cuda(), off.cuda(), lab.cuda(), logit.cuda(), 1.0, 1.0, dirty, loss, 3)
    assert torch.equal(clean[[0, 2]], dirty[[0, 2]]) and bool(torch.isnan(dirty[1]).all()) and math.isnan(float(loss))
    L.policy_loss_grad(out.cuda(), off.cuda(), lab.cuda(), logit.cuda(), None, logit.cuda(), 0.2, 0.2, 0.0, 1.0, dirty, None, loss, 3)
    assert bool(torch.isnan(dirty[1]).all()) and not bool(torch.isnan(dirty[[0, 2]]).any()) and math.isnan(float(loss))
    L.close()


@pytest.mark.parametrize("kind", ["distill", "policy"])
def test_gradients_against_differences(kind):
    """Differences of the loss along random ways: h^2 / 6 of the third derivative (below 4 of the gradient's size for softmaxes of scores of this spread, T >= 1) and the loss's
    own rounding, 2^-24 of it over h = 2^-5."""
    b, m = 4, 300
    off, lab, gen = lists(b, m, [5, 1, 9, 3], 8)
    out = torch.randn(b, m, generator=gen)
    old, ref, adv = policy_values(out, off, lab, gen)
    L = layer(m, b)
    dev = [t.cuda() for t in (off, lab, old, ref, adv)]

    def f(o, g=None):
        loss = torch.empty(1, device="cuda")
        if kind == "distill":
            L.distill_loss_grad(o, dev[0], dev[1], dev[2], 1.5, 1.0, g, loss, b)
        else:
            L.policy_loss_grad(o, *dev, 1.0, 50.0, 0.3, 1.0, g, None, loss, b)   # (bounds that no ratio here reaches: no kink on the way)
        return float(loss)

    o = out.cuda()
    g = torch.empty_like(o)
    base = f(o, g)
    h = 2.0 ** -5
    for n in range(4):
        way = torch.randn(b, m, device="cuda")
        if n % 2:   # along the entries
            way.zero_()
            for i in range(b):
                way[i, lab[off[i]:off[i + 1]].long().cuda()] = torch.randn(int(off[i + 1] - off[i]), device="cuda")
        way /= way.norm()
        diff = (f(o + h * way) - f(o - h * way)) / (2 * h)
        mine = float((g.double() * way.double()).sum())
        assert abs(diff - mine) <= h * h * 4 / 6 * float(g.norm()) * 2 + 4 * R.U * abs(base) / h + 1e-5, (diff, mine)
    L.close()


@pytest.mark.parametrize("m", [10001, 70001])
def test_batches_in_turn_equal_bits_and_a_graph(m):
    s = torch.cuda.Stream()
    b = 6
    off, lab, gen = lists(b, m, [5, 0, 60, 1, 300, 2], 4)
    out = (torch.randn(b, m, generator=gen) * 2).cuda()
    off, lab = off.cuda(), lab.cuda()
    vals = [torch.randn(lab.numel(), generator=gen).cuda() for _ in range(3)]
    L = layer(m, b, s.cuda_stream)

    def make():
        return [torch.full((b, m), math.nan, device="cuda"), torch.full((1,), math.nan, device="cuda"), torch.full((b, m), math.nan, device="cuda"),
                torch.full((lab.numel(),), math.nan, device="cuda"), torch.full((1,), math.nan, device="cuda")]

    def call(o, n=b):
        L.distill_loss_grad(out, off, lab, vals[0], 2.0, 0.1, o[0], o[1], n)
        L.policy_loss_grad(out, off, lab, vals[0], vals[1], vals[2], 0.2, 0.2, 0.1, 0.1, o[2], o[3], o[4], n)

    eager, mine, fewer = make(), make(), make()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call(eager)
        call(fewer, 3)   # a shorter batch: the rows behind it are left as they were
    s.synchronize()
    assert torch.equal(fewer[0][:3], eager[0][:3]) and bool(torch.isnan(fewer[0][3:]).all()) and bool(torch.isnan(fewer[2][3:]).all())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(mine)
    for turn in range(3):
        with torch.cuda.stream(s):
            out.copy_(torch.randn(b, m, device="cuda"))
            for o in mine:
                o.fill_(math.nan)
            g.replay()
            call(fewer, 3)
            call(eager)
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, mine)), turn
    del g
    L.close()
