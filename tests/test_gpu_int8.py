"""8-bit codes to the bit, and products in 8-bit integers against float64."""
import math

import pytest
import torch

import dense_reference as R
from test_gpu_gated import TYPES, check, guarded, untouched, usl

pytestmark = pytest.mark.gpu


def layer(d, b, storage):
    return usl().Layer(3, d, 1, b, storage, torch.cuda.current_stream().cuda_stream)


def quantized(L, rows, shift=0):
    n, w = rows.shape
    store = torch.full((n * w + 512 + shift,), 77, dtype=torch.int8, device="cuda")
    codes = store[256 + shift:256 + shift + n * w].view(n, w)
    scales, ss = guarded(n)
    L.quantize_i8(rows, n, w, codes, scales)
    assert untouched(scales, ss)
    edge = store.clone()
    edge[256 + shift:256 + shift + n * w] = 77
    assert bool((edge == 77).all())
    return codes, scales


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n,w", [(1, 1), (3, 2), (5, 15), (4, 16), (7, 255), (2, 256), (3, 257), (6, 1000), (2, 4099), (1, 65536), (1000, 33), (5, 2048), (5, 2049), (3, 511), (6, 513), (9, 8)])
def test_codes(n, w, storage):
    gen = torch.Generator(device="cuda").manual_seed(n + w)
    rows = (torch.randn(n, w, device="cuda", generator=gen) * torch.exp(4 * torch.randn(n, 1, device="cuda", generator=gen))).to(TYPES[storage])
    L = layer(8, 4, storage)
    for shift in (0, 1):
        codes, scales = quantized(L, rows, shift)
        want_codes, want_scales = R.codes(rows)
        assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), want_codes)
    L.close()


def test_codes_of_ties_zeros_and_the_ends():
    """Halves go to the even code; rows of zeros, of numbers too small for a scale, of the largest numbers; NaN and infinities."""
    w = 256
    half = torch.zeros(w)
    half[:127] = torch.arange(127) + 0.5
    half[127] = 127.0   # scale 1
    half[128:200] = -half[:72]
    rows = [half, torch.zeros(w), torch.full((w,), 1e-45), torch.full((w,), 3.4028234e38), torch.full((w,), -1.0), half.clone(), half.clone(), half.clone()]
    rows[5][3], rows[6][200], rows[7][255] = math.nan, math.inf, -math.inf
    rows = torch.stack(rows).cuda()
    L = layer(8, 4, "f32")
    codes, scales = quantized(L, rows)
    want_codes, want_scales = R.codes(rows)
    assert torch.equal(codes.cpu(), want_codes)
    assert torch.equal(scales[:5].cpu(), want_scales[:5]) and bool(torch.isnan(scales[5:]).all())
    assert codes[0, :4].tolist() == [0, 2, 2, 4] and bool((codes[1:3] == 0).all()) and bool((codes[3] == 127).all()) and bool((codes[4] == -127).all())
    L.close()


def product(q, s, V, t):
    """Exact sums times the scales; the bound: three roundings to float32 beside the last one (an integer's, the scales' product, the product's)."""
    v = (q.double().cpu() @ V.double().cpu().t()) * (s.double().cpu()[:, None] * t.double().cpu())
    return v, 4 * R.U * v.abs()


def numbers(rows, w, seed, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    store = torch.zeros(rows * w + 64 + shift, dtype=torch.int8, device="cuda")
    q = store[shift:shift + rows * w].view(rows, w)
    q.copy_(torch.randint(-127, 128, (rows, w), device="cuda", generator=gen).to(torch.int8))
    return q, torch.rand(rows, device="cuda", generator=gen) * w ** -0.5 / 64


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d,shift", [(1, 1, 1, 0), (1, 64, 16, 0), (2, 63, 17, 0), (16, 65, 15, 1), (16, 1024, 100, 0), (17, 128, 64, 0), (33, 127, 65, 3), (70, 129, 200, 0),
                                         (130, 48, 300, 16), (5, 750, 70, 0), (64, 750, 64, 2), (1, 65536, 5, 0), (20, 65536, 20, 0), (140, 96, 16500, 0), (9, 80, 33000, 0), (16, 256, 16400, 0), (130, 64, 65600, 0), (300, 100, 65601, 0),
                                         (300, 36, 33000, 4), (70, 100, 3001, 0), (70, 1004, 500, 8), (200, 68, 9000, 0)])
def test_products(b, w, d, shift, storage):
    dtype = TYPES[storage]
    q, s = numbers(b, w, 1, shift)
    V, t = numbers(d, w, 2, shift)
    U, u = numbers(d, w, 3, shift)
    if w == 65536:   # the largest sums there are
        q.fill_(127)
        V.fill_(-127)
    L = layer(d, b, storage)
    h, hs = guarded(b, d, dtype=dtype)
    L.project_i8(q, s, V, t, w, h, b)
    want, off = product(q, s, V, t)
    check(h, want, off + R.HALF_STEP[dtype] * (want.abs() + off), "h")
    assert untouched(h, hs)
    for act in (0, 1):
        x, xs = guarded(b, d, dtype=dtype)
        L.gated_block_i8(q, s, V, t, U, u, w, act, x, b)
        (a, da), (p, dp) = product(q, s, V, t), product(q, s, U, u)
        want = R.act(a, act) * p
        off = (1.13 * da + 8 * R.U * a.abs()) * (p.abs() + dp) + R.act(a, act).abs() * dp + 2 * R.U * want.abs()
        check(x, want, off + R.HALF_STEP[dtype] * (want.abs() + off), "x")
        assert untouched(x, xs)
    L.close()


@pytest.mark.parametrize("b", [3, 40])
def test_a_row_that_is_not_a_number_stays_alone(b):
    rows = torch.randn(b, 100, device="cuda")
    rows[1, 50] = math.inf
    V, t = numbers(70, 100, 2)
    L = layer(70, b, "f32")
    codes, scales = quantized(L, rows)
    h = torch.empty(b, 70, device="cuda")
    L.project_i8(codes, scales, V, t, 100, h, b)
    bad = torch.isnan(h).all(1)
    assert bool(bad[1]) and int(torch.isnan(h).any(1).sum()) == 1
    L.close()


def test_a_graph_replayed():
    s = torch.cuda.Stream()
    b, w, d = 40, 200, 300
    V, t = numbers(d, w, 2)
    U, u = numbers(d, w, 3)
    e = torch.randn(b, w, device="cuda")
    L = usl().Layer(3, d, 1, b, "f32", s.cuda_stream)
    codes, scales = torch.empty(b, w, dtype=torch.int8, device="cuda"), torch.empty(b, device="cuda")

    def call(h, x):
        L.quantize_i8(e, b, w, codes, scales)
        L.project_i8(codes, scales, V, t, w, h, b)
        L.gated_block_i8(codes, scales, V, t, U, u, w, 1, x, b)

    eager, mine = ([torch.full((b, d), math.nan, device="cuda") for _ in range(2)] for _ in range(2))
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call(*eager)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(*mine)
    for turn in range(3):
        with torch.cuda.stream(s):
            e.copy_(torch.randn(b, w, device="cuda"))
            for o in mine:
                o.fill_(math.nan)
            g.replay()
            call(*eager)
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, mine)), turn
    del g
    L.close()
