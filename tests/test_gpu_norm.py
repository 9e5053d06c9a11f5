"""Layer norm, forward and backward, against its formulas in float64.

Allowances are worst cases of float32 sums, in units of eps = 2^-24: a lane adds at most 64 values one after the other and the workgroup's
sums meet in a tree of at most 10 levels, so a mean over a row is off by at most 80 eps of the mean of its terms' magnitudes (LONG);
elementwise steps round a few times each.  Sums over the instances: one rounding an addition.  bfloat16 results: half an ulp more."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E, LONG = 2.0 ** -24, 80
EPS = 1e-5


@pytest.fixture(scope="module")
def usl():
    from paper_2306_03725_amd import usl as u
    assert torch.cuda.is_available()
    return u


def rows(b, d, storage, seed, offset=0.5, scale=1.0):
    r = np.random.default_rng([b, d, seed])
    h = r.standard_normal((b, d)) * (scale * (0.25 + 2 * r.random((b, 1)))) + offset * r.standard_normal((b, 1))
    t = torch.from_numpy(h.astype(np.float32))
    return (t if storage == "f32" else t.to(torch.bfloat16)), r


def f64(t):
    return t.detach().cpu().double().numpy()


def reference(h, gamma, beta, eps):
    mean = h.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((h - mean) ** 2).mean(1, keepdims=True) + eps)
    n = (h - mean) * rstd
    return mean, rstd, n, n * gamma + beta


def check(what, got, want, allow):
    got = f64(got)
    assert np.isfinite(got).all(), what
    worst = float((np.abs(got - want) / np.maximum(allow, 1e-300)).max())
    assert worst <= 1.0, "%s: %.3g of what it may be off" % (what, worst)


# one value and few; a wavefront's share and one more; rows that begin at no multiple of 16 bytes; every register form and the widths around its ends; rows beyond them
WIDTHS = [1, 2, 3, 7, 8, 64, 65, 127, 128, 200, 256, 257, 512, 513, 1000, 1003, 1024, 1025, 2048, 2049, 4096, 4100, 5001, 8192, 8193, 10007, 16384, 16385, 30000,
          32768, 32769, 40001, 65536, 65537, 100003]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward(usl, d, storage):
    b = 5
    print("layer norm", b, d, storage, flush=True)
    h, r = rows(b, d, storage, 1)
    gamma, beta = (torch.from_numpy(v.astype(np.float32)) for v in (1 + 0.3 * r.standard_normal(d), r.standard_normal(d)))
    kept = h.dtype
    L = usl.Layer(1, d, 1, 8, storage)
    # guards around the results: nothing beside them is written
    x = torch.full((b * d + 64,), 7.0, dtype=kept, device="cuda")
    mean, rstd = torch.full((b + 8,), 7.0, device="cuda"), torch.full((b + 8,), 7.0, device="cuda")
    L.layer_norm(h.cuda(), gamma.cuda(), beta.cuda(), EPS, x, mean, rstd, b)
    check_forward(h, gamma, beta, EPS, x[:b * d].view(b, d), mean[:b], rstd[:b], storage)
    assert (x[b * d:] == 7).all() and (mean[b:] == 7).all() and (rstd[b:] == 7).all()


def check_forward(h, gamma, beta, eps, x, mean, rstd, storage):
    hd, g, bt = f64(h), f64(gamma), f64(beta)
    m64, r64, n, want = reference(hd, g, bt, eps)
    size = np.abs(hd).mean(1, keepdims=True)          # the mean is off by LONG of this
    off = E * LONG * size
    if mean is not None:
        check("mean", mean, m64[:, 0], (off + E * np.abs(m64))[:, 0] + 1e-300)
    # the variance: LONG of itself, and what the mean's error adds (its square, and deviations that do not add up to zero)
    var = ((hd - m64) ** 2).mean(1, keepdims=True)
    dev = E * (LONG + 8) * var + off * off + 2 * off * np.abs(hd - m64).mean(1, keepdims=True) * E * LONG
    rel = 0.5 * dev / (var + eps) + 4 * E
    if rstd is not None:
        check("rstd", rstd, r64[:, 0], (rel * r64)[:, 0])
    allow = ((off + E * (np.abs(hd) + np.abs(m64))) * r64 + np.abs(n) * (rel + 2 * E)) * np.abs(g) + 2 * E * (np.abs(n * g) + np.abs(bt) + np.abs(want))
    if storage == "bf16":
        allow = allow * (1 + 2.0 ** -8) + np.exp2(np.frexp(want)[1] - 9.0) + 2.0 ** -134   # 8 bits: half an ulp of a value in [2^(e-1), 2^e) is 2^(e-9)
    check("x", x, want, allow + 1e-300)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,d", [(1, 32768), (300, 64), (257, 1003), (1024, 256), (3, 16384), (4099, 96), (65535, 8)])
def test_forward_batches_without_weight_or_statistics(usl, b, d, storage):
    print("layer norm", b, d, storage, flush=True)
    h, r = rows(b, d, storage, 2)
    one, zero = torch.ones(d), torch.zeros(d)
    L = usl.Layer(1, d, 1, b, storage)
    x = torch.empty((b, d), dtype=h.dtype, device="cuda")
    L.layer_norm(h.cuda(), None, None, EPS, x, None, None, b)
    check_forward(h, one, zero, EPS, x, None, None, storage)
    again = h.cuda()
    L.layer_norm(again, None, None, EPS, again, None, None, b)      # in place
    assert torch.equal(again, x)
    g = torch.from_numpy((1 + r.standard_normal(d)).astype(np.float32))
    L.layer_norm(h.cuda(), g.cuda(), None, EPS, x, None, None, b)
    check_forward(h, g, zero, EPS, x, None, None, storage)
    L.layer_norm(h.cuda(), None, g.cuda(), EPS, x, None, None, b)
    check_forward(h, one, g, EPS, x, None, None, storage)


def test_rows_far_from_zero_and_constant_rows(usl):
    """A row around 1000 with deviations of 1: squares around zero would lose the variance.  Constant rows: the deviations are 0 (or the mean's last bit)."""
    b, d = 4, 5000
    h, r = rows(b, d, "f32", 3, offset=0.0, scale=1.0)
    h[0] += 1000.0
    h[1] = 3.0
    h[2] = 0.0
    gamma, beta = torch.ones(d), torch.zeros(d)
    L = usl.Layer(1, d, 1, b)
    x, mean, rstd = torch.empty((b, d), device="cuda"), torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    L.layer_norm(h.cuda(), gamma.cuda(), beta.cuda(), EPS, x, mean, rstd, b)
    check_forward(h, gamma, beta, EPS, x, mean, rstd, "f32")
    assert (x[2] == 0).all()


@pytest.mark.parametrize("d", [96, 5000, 70000])
def test_a_row_that_is_not_finite_stays_alone(usl, d):
    b = 6
    h, _ = rows(b, d, "f32", 4)
    h[1, d // 2] = float("inf")
    h[3, d - 1] = float("nan")
    g = torch.ones(d)
    L = usl.Layer(1, d, 1, b)
    x, mean, rstd = torch.empty((b, d), device="cuda"), torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    L.layer_norm(h.cuda(), None, None, EPS, x, mean, rstd, b)
    assert torch.isnan(x[[1, 3]]).all()
    keep = [0, 2, 4, 5]
    check_forward(h[keep], g, torch.zeros(d), EPS, x[keep], mean[keep], rstd[keep], "f32")


def check_backward(grad_x, h, gamma, mean, rstd, grad_h, grad_gamma, grad_beta):
    hd, gx, g = f64(h), f64(grad_x), f64(gamma)
    m, r = f64(mean)[:, None], f64(rstd)[:, None]
    n, u = (hd - m) * r, gx * g
    mu, mn = u.mean(1, keepdims=True), (u * n).mean(1, keepdims=True)
    want = r * (u - mu - n * mn)
    allow = E * r * (8 * np.abs(u) + (LONG + 8) * np.abs(u).mean(1, keepdims=True) + (LONG + 16) * np.abs(n) * np.abs(u * n).mean(1, keepdims=True))
    check("grad_h", grad_h, want, allow + 1e-300)
    b = len(hd)
    if grad_gamma is not None:
        check("grad_gamma", grad_gamma, (gx * n).sum(0), E * (b + 8) * np.abs(gx * n).sum(0) + 1e-300)
    if grad_beta is not None:
        check("grad_beta", grad_beta, gx.sum(0), E * (b + 8) * np.abs(gx).sum(0) + 1e-300)


def backward(usl, b, d, storage, seed, with_gamma=True, with_beta=True, max_b=None):
    h, r = rows(b, d, storage, seed)
    gamma = torch.from_numpy((1 + 0.3 * r.standard_normal(d)).astype(np.float32))
    grad_x = torch.from_numpy((r.standard_normal((b, d)) / b).astype(np.float32))
    h32 = h.float()
    mean = h32.mean(1)
    rstd = 1.0 / torch.sqrt(((h32 - mean[:, None]) ** 2).mean(1) + EPS)
    L = usl.Layer(1, d, 1, max_b or b, storage)
    grad_h = torch.full((b * d + 64,), 7.0, device="cuda")
    gg, gb = (torch.full((d + 64,), 7.0, device="cuda") if w else None for w in (with_gamma, with_beta))
    L.layer_norm_backward(grad_x.cuda(), h.cuda(), gamma.cuda(), mean.cuda(), rstd.cuda(), grad_h, gg, gb, b)
    assert (grad_h[b * d:] == 7).all() and all((t[d:] == 7).all() for t in (gg, gb) if t is not None)
    check_backward(grad_x, h, gamma, mean, rstd, grad_h[:b * d].view(b, d), gg[:d] if with_gamma else None, gb[:d] if with_beta else None)
    return grad_h, gg, gb


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward_widths(usl, d, storage):
    print("layer norm backward", 9, d, storage, flush=True)
    backward(usl, 9, d, storage, 5)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,d", [(1, 1), (1, 32768), (2, 7), (256, 32768), (4099, 1003), (65535, 8), (33000, 128), (5000, 2048), (700, 16384), (64, 65536), (20000, 96)])
def test_backward_batches(usl, b, d, storage):
    print("layer norm backward", b, d, storage, flush=True)
    backward(usl, b, d, storage, 6)


@pytest.mark.parametrize("b,d", [(40, 1000), (30, 40000)])
def test_backward_without_a_weights_gradient_and_bits(usl, b, d):
    full = backward(usl, b, d, "f32", 7)
    again = backward(usl, b, d, "f32", 7, max_b=4 * b)                       # room for a larger batch: the same bits
    assert all(torch.equal(x, y) for x, y in zip(full, again))
    for gamma, beta in ((True, False), (False, True), (False, False)):
        got = backward(usl, b, d, "f32", 7, gamma, beta)
        assert all(x is None or torch.equal(x, y) for x, y in zip(got, full))


def test_backward_without_a_weight(usl):
    b, d = 7, 300
    h, r = rows(b, d, "f32", 8)
    grad_x = torch.from_numpy(r.standard_normal((b, d)).astype(np.float32))
    mean, rstd = h.mean(1), 1.0 / torch.sqrt(h.var(1, unbiased=False) + EPS)
    L = usl.Layer(1, d, 1, b)
    grad_h = torch.empty((b, d), device="cuda")
    L.layer_norm_backward(grad_x.cuda(), h.cuda(), None, mean.cuda(), rstd.cuda(), grad_h, None, None, b)
    check_backward(grad_x, h, torch.ones(d), mean, rstd, grad_h, None, None)


@pytest.mark.parametrize("b,d", [(3, 17), (6, 700), (4, 40000)])
def test_gradients_against_differences(usl, b, d):
    """Along a random direction the gradients give the slope of sum(grad_x * x), which float64 differences of the formula give too.  Step s: the
    third derivative's share is of the order of s^2 of the terms' magnitudes; the gradients' own share is theirs in check_backward, summed."""
    h, r = rows(b, d, "f32", 9)
    gamma, beta = (r.standard_normal(d).astype(np.float32) for _ in range(2))
    grad_x = r.standard_normal((b, d)).astype(np.float32)
    L = usl.Layer(1, d, 1, b)
    x, mean, rstd = torch.empty((b, d), device="cuda"), torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    gd = torch.from_numpy(gamma).cuda()
    L.layer_norm(h.cuda(), gd, torch.from_numpy(beta).cuda(), EPS, x, mean, rstd, b)
    grad_h, gg, gb = torch.empty((b, d), device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    L.layer_norm_backward(torch.from_numpy(grad_x).cuda(), h.cuda(), gd, mean, rstd, grad_h, gg, gb, b)
    hd, s = f64(h), 1e-4

    def total(dh, dg, db):
        return float((grad_x.astype(np.float64) * reference(hd + dh, gamma.astype(np.float64) + dg, beta.astype(np.float64) + db, EPS)[3]).sum())

    for part, grad in (("h", grad_h), ("gamma", gg), ("beta", gb)):
        way = r.standard_normal(f64(grad).shape)
        zero = {"h": 0.0, "gamma": 0.0, "beta": 0.0}
        slope = (total(*dict(zero, **{part: s * way}).values()) - total(*dict(zero, **{part: -s * way}).values())) / (2 * s)
        got = float((f64(grad) * way).sum())
        size = float((np.abs(f64(grad)) * np.abs(way)).sum()) + float((np.abs(grad_x) * np.abs(gamma)).mean()) * np.abs(way).sum()
        assert abs(got - slope) <= (4 * LONG * E + 100 * s * s) * size, (part, got, slope, size)
