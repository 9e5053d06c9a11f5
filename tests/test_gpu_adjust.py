"""Scores after penalties, bias and mask against float64, and the best labels against a ranking of the scores that the library writes itself.

A score is rounded at most five times on its way (division or product, the penalty's product and sum, its subtraction, the bias): 5 eps of the
largest value on the way."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24


@pytest.fixture(scope="module")
def usl():
    from paper_2306_03725_amd import usl as u
    assert torch.cuda.is_available()
    return u


def bits(allowed):
    """bool [rows][m] -> int32 words [rows][ceil(m/32)]; bits behind the last label are set, and say nothing"""
    rows, m = allowed.shape
    full = np.ones((rows, (m + 31) // 32 * 32), bool)
    full[:, :m] = allowed
    return np.packbits(full.reshape(rows, -1, 32), axis=2, bitorder="little").view(np.uint32).reshape(rows, -1).view(np.int32)


def problem(b, m, shown, masks, seed, levels=None):
    r = np.random.default_rng([b, m, shown, seed])
    out = r.standard_normal((b, m)).astype(np.float32) if levels is None else r.integers(-levels, levels + 1, (b, m)).astype(np.float32)
    bias = r.standard_normal(m).astype(np.float32) if levels is None else r.integers(-1, 2, m).astype(np.float32)
    lists = [r.integers(0, m, r.integers(0, shown + 1)).astype(np.int32) if shown else np.zeros(0, np.int32) for _ in range(b)]
    for i, l in enumerate(lists):      # repeats
        if len(l) > 3:
            l[: len(l) // 3] = l[0]
    if shown and b > 1:
        lists[1] = lists[1][:0]
    allowed = None if masks == "none" else r.random(((b if masks == "each" else 1), m)) < 0.7
    if allowed is not None and b > 2 and masks == "each":
        allowed[2] = False             # nothing is left
    return out, bias, lists, allowed


def reference(out, bias, lists, allowed, repeat, presence, frequency):
    z, size = out.astype(np.float64), np.abs(out.astype(np.float64))
    rep = np.float64(np.float32(repeat))
    for i, l in enumerate(lists):
        j, n = np.unique(l[(l >= 0) & (l < out.shape[1])], return_counts=True)
        old = z[i, j]
        pen = np.where(old > 0, old / rep, old * rep)
        less = np.float64(np.float32(presence)) + np.float64(np.float32(frequency)) * n
        size[i, j] = np.maximum(size[i, j], np.abs(pen)) + np.abs(np.float64(np.float32(presence))) + np.abs(np.float64(np.float32(frequency))) * n
        z[i, j] = pen - less
    if bias is not None:
        z, size = z + bias, size + np.abs(bias)
    if allowed is not None:
        z = np.where(allowed, z, -np.inf)
    return z, size


def adjustments(usl, bias, lists, allowed, **scalars):
    off = np.concatenate([[0], np.cumsum([len(l) for l in lists])]).astype(np.int64)
    lab = np.concatenate(lists).astype(np.int32)
    return usl.Adjustments(bias=None if bias is None else torch.from_numpy(bias).cuda(), allowed=None if allowed is None else torch.from_numpy(bits(allowed)).cuda(),
                           shown_off=torch.from_numpy(off).cuda(), shown_lab=torch.from_numpy(lab).cuda(), **scalars)


def adjusted(usl, L, out, a):
    b, m = out.shape
    got = torch.full((b * m + 64,), 7.0, device="cuda")
    dev = torch.from_numpy(out).cuda()
    L.adjust_scores(dev, a, got, b)
    assert (got[b * m:] == 7).all()
    L.adjust_scores(dev, a, dev, b)                      # in place: the same bits
    assert torch.equal(dev.view(torch.int32), got[:b * m].view(b, m).view(torch.int32))
    return got[:b * m].view(b, m).cpu().numpy()


def ranked(z, allowed, kk):
    b, m = z.shape
    lab, val = np.full((b, kk), -1, np.int32), np.full((b, kk), -np.inf, np.float32)
    for i in range(b):
        j = np.arange(m) if allowed is None else np.nonzero(np.broadcast_to(allowed, (b, m))[i])[0]
        j = j[np.lexsort((j, -(z[i, j] + 0.0)))][:kk]
        lab[i, :len(j)], val[i, :len(j)] = j, z[i, j]
    return lab, val


def best(usl, L, out, a, kk):
    b = out.shape[0]
    lab = torch.full((b * kk + 8,), 77, dtype=torch.int32, device="cuda")
    val = torch.full((b * kk + 8,), 77.0, device="cuda")
    L.topk_adjusted(torch.from_numpy(out).cuda(), a, b, kk, lab, val)
    assert (lab[b * kk:] == 77).all() and (val[b * kk:] == 77).all()
    return lab[:b * kk].view(b, kk).cpu().numpy(), val[:b * kk].view(b, kk).cpu().numpy()


PENALTIES = dict(repeat=1.3, presence=0.25, frequency=0.125)
SIZES = [(1, 1, 3), (2, 5, 4), (4, 31, 10), (3, 33, 200), (5, 1000, 0), (6, 2047, 50), (1, 2049, 2000), (3, 8191, 300), (2, 8193, 9000), (40, 3001, 70), (7, 70001, 500), (1, 500000, 200),
         (2, 1000003, 20000), (300, 30938, 40), (60, 100002, 300)]


@pytest.mark.parametrize("masks", ["none", "one", "each"])
@pytest.mark.parametrize("b,m,shown", SIZES)
def test_adjust_and_rank(usl, b, m, shown, masks):
    print("adjust", b, m, shown, masks, flush=True)
    out, bias, lists, allowed = problem(b, m, shown, masks, 1)
    L = usl.Layer(m, 1, 1, b)
    a = adjustments(usl, bias, lists, allowed, **PENALTIES)
    got = adjusted(usl, L, out, a)
    want, size = reference(out, bias, lists, allowed, **PENALTIES)
    finite = np.isfinite(want)
    assert (np.isneginf(got) == ~finite).all()
    assert (np.abs(got[finite].astype(np.float64) - want[finite]) <= 5 * E * size[finite]).all()
    for kk in (1, 5, 32):
        if kk <= m:
            lab, val = best(usl, L, out, a, kk)
            ref_lab, ref_val = ranked(got, allowed, kk)
            np.testing.assert_array_equal(lab, ref_lab)
            np.testing.assert_array_equal(val.view(np.uint32), ref_val.view(np.uint32))


@pytest.mark.parametrize("b,m,shown,kk", [(3, 3000, 400, 32), (50, 20000, 3000, 17), (1, 40000, 100, 5)])
def test_equal_scores_rank_by_label(usl, b, m, shown, kk):
    """Few distinct values, exact in float32: the ranking has ties everywhere, also with the shown labels'."""
    out, bias, lists, allowed = problem(b, m, shown, "each", 2, levels=2)
    L = usl.Layer(m, 1, 1, b)
    a = adjustments(usl, bias, lists, allowed, repeat=2.0, presence=0.5, frequency=0.5)
    got = adjusted(usl, L, out, a)
    want, _ = reference(out, bias, lists, allowed, 2.0, 0.5, 0.5)
    np.testing.assert_array_equal(got, want.astype(np.float32))
    lab, val = best(usl, L, out, a, kk)
    ref_lab, ref_val = ranked(got, allowed, kk)
    np.testing.assert_array_equal(lab, ref_lab)
    np.testing.assert_array_equal(val, ref_val)


@pytest.mark.parametrize("m,left", [(500, 0), (500, 3), (20000, 1), (20000, 7), (300000, 4)])
def test_masks_that_leave_few(usl, m, left):
    """Fewer allowed labels than are asked for: they are listed, then label -1 and -infinity; an allowed score of -infinity is a score."""
    r = np.random.default_rng([m, left])
    b, kk = 3, 8
    out = r.standard_normal((b, m)).astype(np.float32)
    allowed = np.zeros((b, m), bool)
    for i in range(b):
        allowed[i, r.choice(m, left, replace=False)] = True
    if left:
        out[0, np.nonzero(allowed[0])[0][0]] = -np.inf
    L = usl.Layer(m, 1, 1, b)
    a = usl.Adjustments(allowed=torch.from_numpy(bits(allowed)).cuda())
    lab, val = best(usl, L, out, a, kk)
    ref_lab, ref_val = ranked(np.where(allowed, out, -np.inf).astype(np.float32), allowed, kk)
    np.testing.assert_array_equal(lab, ref_lab)
    np.testing.assert_array_equal(val, ref_val)


def test_masked_scores_may_be_anything(usl):
    """NaN, infinities and the type's lowest value where the mask hides them; infinities and the lowest value as scores."""
    b, m, kk = 4, 9001, 6
    r = np.random.default_rng(5)
    out = r.standard_normal((b, m)).astype(np.float32)
    allowed = np.ones((b, m), bool)
    for v in (np.nan, -np.nan, np.inf, -np.inf, np.finfo(np.float32).min, np.finfo(np.float32).max):
        at = r.integers(0, m, 400)
        for i in range(b):
            out[i, at], allowed[i, at] = v, False
    out[1, 17], allowed[1, 17] = np.inf, True
    out[2, :], allowed[2, :] = np.finfo(np.float32).min, True
    out[3, 4000], allowed[3, 4000] = -np.inf, True
    L = usl.Layer(m, 1, 1, b)
    lists = [np.arange(0, m, 7, dtype=np.int32)] * b                # shown labels among the masked ones too
    a = adjustments(usl, None, lists, allowed, repeat=1.5)
    got = adjusted(usl, L, out, a)
    assert not np.isnan(got).any() and np.isneginf(got[~allowed]).all()
    want, size = reference(np.where(allowed, out, 0).astype(np.float32), None, lists, allowed, 1.5, 0.0, 0.0)
    with np.errstate(invalid="ignore", over="ignore"):
        ok = allowed & np.isfinite(want) & (np.abs(want) <= np.finfo(np.float32).max)
        assert (np.abs(got[ok].astype(np.float64) - want[ok]) <= 5 * E * size[ok]).all()
    assert got[1, 17] == np.inf and got[3, 4000] == -np.inf
    lab, val = best(usl, L, out, a, kk)
    ref_lab, ref_val = ranked(got, allowed, kk)
    np.testing.assert_array_equal(lab, ref_lab)
    np.testing.assert_array_equal(val, ref_val)
    assert lab[1, 0] == 17


def test_entries_outside_the_labels_say_nothing(usl):
    b, m = 2, 5000
    out, bias, lists, _ = problem(b, m, 50, "none", 6)
    lists = [np.concatenate([l, np.array([-1, m, -2 ** 31, 2 ** 31 - 1, m + 7], np.int32)]) for l in lists]
    L = usl.Layer(m, 1, 1, b)
    got = adjusted(usl, L, out, adjustments(usl, bias, lists, None, **PENALTIES))
    want, size = reference(out, bias, lists, None, **PENALTIES)
    assert (np.abs(got.astype(np.float64) - want) <= 5 * E * size).all()


def test_nothing_to_adjust_and_labels_shown_often(usl):
    b, m = 3, 10000
    out, bias, lists, _ = problem(b, m, 0, "none", 7)
    L = usl.Layer(m, 1, 1, b)
    got = adjusted(usl, L, out, usl.Adjustments())
    assert (got.view(np.uint32) == out.view(np.uint32)).all()       # to the bit
    empty = adjustments(usl, None, lists, None, **PENALTIES)          # lists without an entry
    assert (adjusted(usl, L, out, empty).view(np.uint32) == out.view(np.uint32)).all()
    lab, val = best(usl, L, out, usl.Adjustments(), 9)
    ref_lab, ref_val = ranked(out, None, 9)
    np.testing.assert_array_equal(lab, ref_lab)
    lists = [np.full(100000, 4321, np.int32), np.zeros(1, np.int32), np.arange(m, dtype=np.int32).repeat(11)]
    got = adjusted(usl, L, out, adjustments(usl, bias, lists, None, **PENALTIES))
    want, size = reference(out, bias, lists, None, **PENALTIES)
    assert (np.abs(got.astype(np.float64) - want) <= 5 * E * size).all()


def test_more_masks_than_instances_and_a_smaller_batch(usl):
    m, most = 20001, 8
    out, bias, lists, allowed = problem(most, m, 90, "each", 8)
    L = usl.Layer(m, 1, 1, most)
    whole = adjusted(usl, L, out, adjustments(usl, bias, lists, allowed, **PENALTIES))
    for b in (1, 5):
        a = usl.Adjustments(bias=torch.from_numpy(bias).cuda(), allowed=torch.from_numpy(bits(allowed)).cuda(), **PENALTIES,
                            shown_off=torch.from_numpy(np.concatenate([[0], np.cumsum([len(l) for l in lists])]).astype(np.int64)).cuda(),
                            shown_lab=torch.from_numpy(np.concatenate(lists)).cuda())
        assert (adjusted(usl, L, out[:b], a).view(np.uint32) == whole[:b].view(np.uint32)).all()


def test_rows_that_begin_anywhere(usl):
    """Scores, results and bias at addresses that are multiples of 4 bytes only."""
    b, m = 3, 8197
    out, bias, lists, allowed = problem(b, m, 60, "each", 9)
    L = usl.Layer(m, 1, 1, b)
    a = adjustments(usl, bias, lists, allowed, **PENALTIES)
    want = adjusted(usl, L, out, a)
    for shift in (1, 2, 3):
        src, dst = torch.zeros(b * m + 8, device="cuda"), torch.zeros(b * m + 8, device="cuda")
        base = torch.zeros(m + 8, device="cuda")
        src[shift:shift + b * m] = torch.from_numpy(out).cuda().view(-1)
        base[shift:shift + m] = torch.from_numpy(bias).cuda()
        a2 = adjustments(usl, None, lists, allowed, **PENALTIES)
        a2._a.bias = base.data_ptr() + 4 * shift
        L.adjust_scores(src.data_ptr() + 4 * shift, a2, dst.data_ptr() + 4 * (4 - shift), b)
        torch.cuda.synchronize()
        got = dst[4 - shift:4 - shift + b * m].view(b, m).cpu().numpy()
        assert (got.view(np.uint32) == want.view(np.uint32)).all()


def test_another_stream_and_a_graph(usl):
    b, m, kk = 2, 60000, 5
    out, bias, lists, allowed = problem(b, m, 100, "each", 10)
    a = adjustments(usl, bias, lists, allowed, **PENALTIES)
    dev = torch.from_numpy(out).cuda()
    lab, val, got = torch.empty((b, kk), dtype=torch.int32, device="cuda"), torch.empty((b, kk), device="cuda"), torch.empty((b, m), device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    L = usl.Layer(m, 1, 1, b, "f32", s.cuda_stream)

    def call():
        L.adjust_scores(dev, a, got, b)
        L.topk_adjusted(dev, a, b, kk, lab, val)

    call()
    s.synchronize()
    want = [t.clone() for t in (lab, val, got)]
    np.testing.assert_array_equal(lab.cpu().numpy(), ranked(got.cpu().numpy(), allowed, kk)[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call()
    for turn in range(3):
        lab.fill_(-5)
        val.fill_(0)
        got.fill_(0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((lab, val, got), want)), turn


# short segments by themselves and runs of long ones, few and many candidates to merge, batches that fill the chip more than once
PATHS = [(6552, 189, 10), (20000, 300, 5), (46472, 92, 1), (58262, 49, 32), (100000, 100, 32), (100001, 1100, 3), (500000, 1, 32), (747351, 57, 5), (1761053, 2, 32), (2900000, 1, 32),
         (4300003, 1, 32), (4096, 1500, 32)]


@pytest.mark.parametrize("order", ["any", "rising", "falling", "equal"])
@pytest.mark.parametrize("m,b,kk", PATHS)
def test_scores_in_any_order(usl, m, b, kk, order):
    """Scores in any order, rising with the label (every segment is better than those before), falling, all equal; against a stable sort."""
    print("order", m, b, kk, order, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(m + kk)
    if order == "any":
        out = torch.randn((b, m), device="cuda", generator=gen)
    elif order == "equal":
        out = torch.full((b, m), 0.5, device="cuda")
    else:
        out = torch.arange(m, device="cuda", dtype=torch.float32).mul_(1.0 if order == "rising" else -1.0).repeat(b, 1)
    words = torch.randint(-2 ** 31, 2 ** 31, ((m + 31) // 32,), device="cuda", generator=gen, dtype=torch.int64).to(torch.int32)
    allowed = ((words[:, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1).view(-1)[:m] != 0
    L = usl.Layer(m, 1, 1, b)
    lab, val = torch.empty((b, kk), dtype=torch.int32, device="cuda"), torch.empty((b, kk), device="cuda")
    for mask in (None, words[None, :]):
        L.topk_adjusted(out, usl.Adjustments(allowed=mask), b, kk, lab, val)
        for i in {0, b // 2, b - 1}:
            z = out[i] if mask is None else torch.where(allowed, out[i], -float("inf"))
            want, at = z.sort(descending=True, stable=True)
            assert torch.equal(lab[i].long(), at[:kk]) and torch.equal(val[i], want[:kk]), (i, mask is None)
    if order != "equal":
        L.topk(out, b, kk, lab, val)
        want, at = out[b - 1].sort(descending=True, stable=True)
        assert torch.equal(lab[b - 1].long(), at[:kk]) and torch.equal(val[b - 1], want[:kk])
