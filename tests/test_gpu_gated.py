"""The gated block and its backward pass against float64, at the sizes where tiles, steps and rows end, at any alignment; chunks of a batch; streams and graphs."""
import pytest
import torch

import dense_reference as R

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GUARD = 64


def usl():
    from paper_2306_03725_amd import usl as u
    return u


def guarded(*shape, dtype=torch.float32, shift=0):
    """A tensor of NaN between guards of NaN, `shift` elements off a multiple of 256 bytes."""
    n = 1
    for s in shape:
        n *= s
    store = torch.full((n + 2 * GUARD * 4 + shift,), float("nan"), dtype=dtype, device="cuda")
    view = store[GUARD * 4 + shift:GUARD * 4 + shift + n].view(shape)
    return view, store


def untouched(view, store):
    flat = store.clone()
    at = (view.data_ptr() - store.data_ptr()) // store.element_size()
    flat[at:at + view.numel()] = float("nan")
    return bool(torch.isnan(flat).all())


def shifted(t, shift):
    v, _ = guarded(*t.shape, dtype=t.dtype, shift=shift)
    return v.copy_(t)


def inputs(b, w, d, dtype, seed=0, shift=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    e = torch.randn(b, w, device="cuda", generator=gen).to(dtype)
    Vg, Vu = ((torch.randn(d, w, device="cuda", generator=gen) * w ** -0.5).to(dtype) for _ in range(2))
    return [shifted(t, shift) for t in (e, Vg, Vu)]


def check(got, want, bound, what):
    got = got.double().cpu()
    err = (got - want).abs()
    room = bound + R.HALF_STEP[torch.float32] * want.abs() + 1e-300
    worst = float((err / room).max())
    assert worst <= 1.0, "%s: worst error over its bound %.3g" % (what, worst)


def forward_case(b, w, d, storage, act, shift=0, keep=True):
    dtype = TYPES[storage]
    e, Vg, Vu = inputs(b, w, d, dtype, seed=b * 7 + w, shift=shift)
    L = usl().Layer(3, d, 1, b, storage, torch.cuda.current_stream().cuda_stream)
    (x, xs), (gate, gs), (up, us) = (guarded(b, d, dtype=dtype, shift=shift) for _ in range(3))
    L.gated_block(e, Vg, Vu, w, act, x, gate if keep else None, up if keep else None, b)
    want = R.gated(e, Vg, Vu, act)
    half = R.HALF_STEP[dtype]
    for got, (value, off), name in zip((gate, up, x), want, ("gate", "up", "x")):
        if keep or name == "x":
            check(got, value, off + half * (value.abs() + off), name)
    assert untouched(x, xs) and untouched(gate, gs) and untouched(up, us)
    L.close()


# around the sizes of fragments, steps, tiles and of the kernels' borders
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d", [(1, 1, 1), (1, 64, 16), (2, 3, 17), (16, 33, 15), (16, 512, 100), (17, 64, 64), (17, 65, 63), (31, 7, 129), (64, 128, 128),
                                   (65, 127, 65), (100, 96, 200), (130, 40, 300), (3, 1000, 70), (1, 2049, 33), (200, 256, 33)])
def test_forward(b, w, d, storage):
    for act in (0, 1):
        forward_case(b, w, d, storage, act)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d,shift", [(5, 64, 64, 1), (5, 64, 64, 2), (5, 24, 40, 4), (70, 64, 130, 1), (70, 64, 130, 3), (70, 48, 64, 8), (40, 72, 66, 0), (40, 71, 68, 1)])
def test_forward_at_any_alignment(b, w, d, shift, storage):
    forward_case(b, w, d, storage, 0, shift=shift)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d", [(130, 64, 16384), (300, 72, 16400), (257, 65, 20000), (200, 136, 32770), (300, 40, 32768), (1, 64, 16384), (16, 200, 16390),
                                   (7, 768, 32769), (15, 8, 16385), (65, 64, 32768), (64, 96, 16400), (257, 64, 33000), (169, 72, 16512),
                                   (700, 40, 9000), (129, 33, 12000), (47, 900, 64), (250, 130, 400)])
def test_forward_of_large_tiles(b, w, d, storage):
    forward_case(b, w, d, storage, 0)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d,shift", [(300, 70, 32770, 0), (300, 30, 32768, 0), (300, 64, 32768, 2), (130, 70, 16400, 0), (257, 201, 20001, 0), (200, 70, 9000, 2), (70, 70, 3001, 0),
                                         (70, 2, 3001, 0), (70, 64, 3001, 2), (100, 130, 1500, 0)])
def test_forward_of_rows_of_words(b, w, d, shift, storage):
    forward_case(b, w, d, storage, b % 2, shift=shift)


@pytest.mark.parametrize("b", [4, 40])
def test_forward_keeps_nothing_if_not_asked(b):
    forward_case(b, 50, 60, "bf16", 1, keep=False)


@pytest.mark.parametrize("b", [3, 50])
def test_forward_of_one_row_does_not_depend_on_the_others(b):
    """An instance with NaN and infinities leaves the others alone."""
    e, Vg, Vu = inputs(b, 96, 70, torch.float32)
    L = usl().Layer(3, 70, 1, b, "f32", torch.cuda.current_stream().cuda_stream)
    x0, x1 = torch.empty(b, 70, device="cuda"), torch.empty(b, 70, device="cuda")
    L.gated_block(e, Vg, Vu, 96, 0, x0, None, None, b)
    e[1, 5], e[1, 6] = float("nan"), float("inf")
    L.gated_block(e, Vg, Vu, 96, 0, x1, None, None, b)
    keep = [i for i in range(b) if i != 1]
    assert torch.equal(x0[keep], x1[keep]) and bool(torch.isnan(x1[1]).all())
    L.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("value", [0.0, -200.0, 200.0])
def test_far_gates(storage, value):
    """act(-200) is 0 (or the number next to it), act(200) is 200: no overflow on the way, forward or backward."""
    dtype = TYPES[storage]
    for act in (0, 1):
        e, Vg, Vu = torch.ones(2, 1, device="cuda").to(dtype), torch.full((8, 1), value, device="cuda").to(dtype), torch.ones(8, 1, device="cuda").to(dtype)
        L = usl().Layer(3, 8, 1, 2, storage, torch.cuda.current_stream().cuda_stream)
        x, gate, up = (torch.empty(2, 8, device="cuda", dtype=dtype) for _ in range(3))
        L.gated_block(e, Vg, Vu, 1, act, x, gate, up, 2)
        assert torch.equal(x.float(), torch.full((2, 8), max(value, 0.0), device="cuda"))
        ge, gg, gu = torch.empty(2, 1, device="cuda"), torch.empty(8, 1, device="cuda"), torch.empty(8, 1, device="cuda")
        L.gated_block_backward(torch.ones(2, 8, device="cuda"), e, Vg, Vu, gate, up, 1, act, ge, gg, gu, 2)
        by_gate = 0.0 if value < 0 else 1.0 if value > 0 else 0.5
        assert torch.equal(gg, torch.full((8, 1), 2 * by_gate, device="cuda"))
        assert torch.equal(gu, torch.full((8, 1), 2 * max(value, 0.0), device="cuda"))
        assert torch.equal(ge, torch.full((2, 1), 8 * (by_gate * value + max(value, 0.0)), device="cuda"))
        L.close()


def backward_case(b, w, d, storage, act, shift=0, layer=None, which=(True, True, True)):
    dtype = TYPES[storage]
    e, Vg, Vu = inputs(b, w, d, dtype, seed=b * 5 + w, shift=shift)
    gen = torch.Generator(device="cuda").manual_seed(3)
    grad_x = shifted(torch.randn(b, d, device="cuda", generator=gen) / b, shift)
    gate, up = (shifted((e.float() @ V.float().t()).to(dtype), shift) for V in (Vg, Vu))
    L = layer or usl().Layer(3, d, 1, b, storage, torch.cuda.current_stream().cuda_stream)
    outs = [guarded(*s, shift=shift) for s in ((b, w), (d, w), (d, w))]
    L.gated_block_backward(grad_x, e, Vg, Vu, gate, up, w, act, *[o[0] if on else None for o, on in zip(outs, which)], b)
    for (got, store), (want, off, norm), name, on in zip(outs, R.gated_backward(grad_x, e, Vg, Vu, gate, up, act), ("grad_e", "grad_V_gate", "grad_V_up"), which):
        assert untouched(got, store), name
        if not on:
            assert bool(torch.isnan(got).all()), name
            continue
        check(got, want, off, name)
        if want.numel() >= 256:
            rel = float((got.double().cpu() - want).norm() / want.norm())
            assert rel <= norm, "%s: norm of the error %.3g, bound %.3g" % (name, rel, norm)
    if layer is None:
        L.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d", [(1, 1, 1), (1, 64, 16), (2, 3, 17), (31, 33, 15), (32, 128, 128), (33, 129, 127), (64, 64, 256), (100, 96, 200), (129, 40, 300),
                                   (7, 300, 1000), (1, 768, 2000), (200, 256, 33)])
def test_backward(b, w, d, storage):
    for act in (0, 1):
        backward_case(b, w, d, storage, act)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d", [(5, 264, 33000), (32, 301, 33000), (33, 264, 33000), (64, 299, 33001), (150, 500, 8100), (130, 384, 16400), (17, 513, 8192),
                                   (161, 264, 33000), (300, 520, 8200), (40, 71, 9001), (20, 334, 9001), (140, 3, 9001), (140, 4, 9001),
                                   (40, 270, 33023), (161, 278, 33100), (9, 302, 33001)])
def test_backward_of_large_tiles(b, w, d, storage):
    backward_case(b, w, d, storage, b % 2)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d,shift", [(5, 64, 64, 1), (70, 64, 130, 2), (70, 48, 64, 4), (40, 71, 68, 1), (40, 130, 66, 8)])
def test_backward_at_any_alignment(b, w, d, shift, storage):
    backward_case(b, w, d, storage, 0, shift=shift)


@pytest.mark.parametrize("which", [(True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, True, False), (False, False, False)])
def test_backward_of_what_is_asked_for(which):
    backward_case(20, 72, 90, "bf16", 0, which=which)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_batches_in_turn(storage):
    """Scratch of another batch or width before: nothing of it is left in the next call's sums."""
    L = usl().Layer(3, 200, 1, 300, storage, torch.cuda.current_stream().cuda_stream)
    for b, w in ((300, 130), (3, 20), (65, 130), (1, 300), (290, 64), (3, 20)):
        backward_case(b, w, 200, storage, 0, layer=L)
    L.close()


def test_batch_in_chunks():
    """More instances than a chunk's scratch has room for: the matrices' gradients are added up over the chunks."""
    d, w, b = 1 << 19, 4, 300   # a row of G takes 6.3 MB: chunks of 256
    backward_case(b, w, d, "bf16", 0)


def test_backward_gives_equal_bits():
    e, Vg, Vu = inputs(100, 200, 3000, torch.bfloat16)
    gate, up = ((e.float() @ V.float().t()).bfloat16() for V in (Vg, Vu))
    grad_x = torch.randn(100, 3000, device="cuda")
    L = usl().Layer(3, 3000, 1, 100, "bf16", torch.cuda.current_stream().cuda_stream)
    runs = []
    for _ in range(3):
        outs = [torch.empty(100, 200, device="cuda"), torch.empty(3000, 200, device="cuda"), torch.empty(3000, 200, device="cuda")]
        L.gated_block_backward(grad_x, e, Vg, Vu, gate, up, 200, 0, *outs, 100)
        runs.append(outs)
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(runs[0], r))
    L.close()


@pytest.mark.parametrize("act", [0, 1])
def test_gradients_against_differences(act):
    """The backward pass against differences of the forward one, float32: (f(v + h) - f(v - h)) / 2h with h = 2^-6 is off by h^2 / 6 of the third
    derivative along the line (below 4 |x| for both activations at these sizes: 2e-4 of the gradient) and by roundings of f, 2^-24 * sqrt(n) / h."""
    b, w, d = 6, 20, 40
    e, Vg, Vu = inputs(b, w, d, torch.float32, seed=11)
    grad_x = torch.randn(b, d, device="cuda")
    L = usl().Layer(3, d, 1, b, "f32", torch.cuda.current_stream().cuda_stream)

    def f(e, Vg, Vu):
        x = torch.empty(b, d, device="cuda")
        L.gated_block(e, Vg, Vu, w, act, x, None, None, b)
        return float((x.double() * grad_x.double()).sum())

    x, gate, up = (torch.empty(b, d, device="cuda") for _ in range(3))
    L.gated_block(e, Vg, Vu, w, act, x, gate, up, b)
    outs = [torch.empty(b, w, device="cuda"), torch.empty(d, w, device="cuda"), torch.empty(d, w, device="cuda")]
    L.gated_block_backward(grad_x, e, Vg, Vu, gate, up, w, act, *outs, b)
    h = 2.0 ** -6
    for n in range(3):
        args = [e, Vg, Vu]
        way = torch.randn_like(args[n])
        way /= way.norm()
        plus, minus = list(args), list(args)
        plus[n], minus[n] = args[n] + h * way, args[n] - h * way
        diff = (f(*plus) - f(*minus)) / (2 * h)
        mine = float((outs[n].double() * way.double()).sum())
        size = float(outs[n].norm())
        assert abs(diff - mine) <= 1e-3 * size + 1e-4, (n, diff, mine, size)
    L.close()


@pytest.mark.parametrize("b,w,d", [(70, 136, 500), (300, 264, 16500), (5, 136, 16500)])
def test_another_stream_and_a_graph(b, w, d):
    """On a stream of its own, captured and replayed with eager calls between: every replay gives the eager call's bits."""
    s = torch.cuda.Stream()
    e, Vg, Vu = inputs(b, w, d, torch.bfloat16, seed=2)
    grad_x = torch.randn(b, d, device="cuda")
    L = usl().Layer(3, d, 1, b, "bf16", s.cuda_stream)

    def make():
        return ([torch.full((b, d), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(3)]
                + [torch.full((b, w), float("nan"), device="cuda")] + [torch.full((d, w), float("nan"), device="cuda") for _ in range(2)])

    def call(o):
        L.gated_block(e, Vg, Vu, w, 0, o[0], o[1], o[2], b)
        L.gated_block_backward(grad_x, e, Vg, Vu, o[1], o[2], w, 0, o[3], o[4], o[5], b)

    eager, mine = make(), make()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call(eager)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call(mine)
    for turn in range(3):
        with torch.cuda.stream(s):
            e.copy_(torch.randn(b, w, device="cuda"))
            for o in mine:
                o.fill_(float("nan"))
            g.replay()
            call(eager)
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(eager, mine)), turn
    del g
    L.close()


def test_a_graph_survives_a_call_that_needs_more_scratch():
    """Captured with a narrow e, then an eager call with a wide one, which needs more scratch than there is: the graph's is still its own."""
    s = torch.cuda.Stream()
    b, d = 40, 300
    L = usl().Layer(3, d, 1, b, "bf16", s.cuda_stream)

    def make(w):
        e, Vg, Vu = inputs(b, w, d, torch.bfloat16, seed=w)
        gate, up = ((e.float() @ V.float().t()).bfloat16() for V in (Vg, Vu))
        o = [torch.full((b, w), float("nan"), device="cuda"), torch.full((d, w), float("nan"), device="cuda"), torch.full((d, w), float("nan"), device="cuda")]
        return (torch.randn(b, d, device="cuda"), e, Vg, Vu, gate, up, w, 0), o

    (narrow, out), (wide, out_wide) = make(64), make(40000)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        L.gated_block_backward(*narrow, *out, b)
    s.synchronize()
    want = [o.clone() for o in out]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        L.gated_block_backward(*narrow, *out, b)
    for _ in range(3):
        with torch.cuda.stream(s):
            L.gated_block_backward(*wide, *out_wide, b)
            for o in out:
                o.fill_(float("nan"))
            g.replay()
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, want))
    with torch.cuda.stream(s):
        L.gated_block_backward(*narrow, *out, b)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(out, want))
    del g
    L.close()
