"""The block, the layer and the losses together, as they are used: one gradient from the loss to e and the matrices against float64; offsets beyond 32 bits; the example."""
import math
import os
import sys

import pytest
import torch

import dense_reference as R
from test_gpu_gated import TYPES, inputs, usl

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("loss_of", ["distill", "policy"])
def test_one_gradient_through_everything(loss_of):
    """e -> gated block -> scores -> loss -> backward products -> the block's backward pass, float32, against float64's automatic gradient of the same function.  Errors: roundings of
    sums of at most 2 d = 600 products in five steps one behind the other, each at most 2^-24 * (16 + sqrt(600)) as a norm, and what softmax and activation add: below 8 * 2^-24 *
    60 of the gradient's norm, 3e-5."""
    b, w, d, m, k, T = 12, 40, 300, 700, 8, 1.5
    e, Vg, Vu = inputs(b, w, d, torch.float32, seed=21)
    L = usl().Layer(m, d, k, b, "f32", torch.cuda.current_stream().cuda_stream)
    idx = torch.empty(m, k, dtype=torch.int32, device="cuda")
    L.init_indices(idx, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    W = torch.randn(m, k, device="cuda", generator=gen)
    lengths = [i % 6 for i in range(b)]
    off = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    n = int(off[-1])
    lab = torch.randint(0, m, (n,), device="cuda", generator=gen).to(torch.int32)
    v = [torch.randn(n, device="cuda", generator=gen) for _ in range(3)]
    x, gate, up = (torch.empty(b, d, device="cuda") for _ in range(3))
    out, loss = torch.empty(b, m, device="cuda"), torch.empty(1, device="cuda")
    L.gated_block(e, Vg, Vu, w, 1, x, gate, up, b)
    L.forward(x, idx, W, out, b)
    row = torch.repeat_interleave(torch.arange(b, device="cuda"), torch.tensor(lengths, device="cuda"))
    lp = torch.log_softmax(out.double(), 1)[row, lab.long()]
    old, ref = (lp + 0.1 * v[1]).float(), (lp + 0.1 * v[2]).float()
    if loss_of == "distill":
        L.distill_loss_grad(out, off, lab, v[0], T, 0.5, out, loss, b)
    else:
        L.policy_loss_grad(out, off, lab, old, ref, v[0], 1.0, 20.0, 0.2, 0.5, out, None, loss, b)
    grad_W, grad_x = torch.empty(m, k, device="cuda"), torch.empty(b, d, device="cuda")
    L.backward(out, x, idx, W, grad_W, grad_x, b)
    got = [torch.empty(b, w, device="cuda"), torch.empty(d, w, device="cuda"), torch.empty(d, w, device="cuda")]
    L.gated_block_backward(grad_x, e, Vg, Vu, gate, up, w, 1, *got, b)
    p = [t.double().cpu().requires_grad_() for t in (e, Vg, Vu, W)]
    a, u = p[0] @ p[1].t(), p[0] @ p[2].t()
    z = ((R.act(a, 1) * u)[:, idx.long().cpu()] * p[3]).sum(2)
    row, at = row.cpu(), lab.long().cpu()
    if loss_of == "distill":
        t = v[0].double().cpu() / T
        log_p = torch.cat([torch.log_softmax(s, 0) for s in t.split(lengths)])
        total = 0.5 * T * T * (torch.exp(log_p) * (log_p - torch.log_softmax(z / T, 1)[row, at])).sum()
    else:
        q, adv = torch.log_softmax(z, 1)[row, at], v[0].double().cpu()
        gap = ref.double().cpu() - q
        total = 0.5 * (0.2 * (torch.exp(gap) - gap - 1) - torch.exp(q - old.double().cpu()) * adv).sum()
    total.backward()
    assert abs(float(loss) - float(total.detach())) <= 3e-5 * (1 + abs(float(total.detach())))
    for mine, want, name in zip(got + [grad_W], p, ("grad_e", "grad_V_gate", "grad_V_up", "grad_W")):
        rel = float((mine.double().cpu() - want.grad).norm() / want.grad.norm())
        assert rel <= 3e-5, (name, rel)
    L.close()


def test_scores_beyond_32_bits():
    """1024 rows of 3 million scores: the gradient of the last rows lies behind 2^31 and 2^33 bytes."""
    b, m = 1024, 3000000
    out = torch.empty(b, m, device="cuda")
    out.normal_()
    lengths = [i % 3 for i in range(b)]
    off = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    n = int(off[-1])
    lab = torch.randint(0, m, (n,), device="cuda").to(torch.int32)
    logit = torch.randn(n, device="cuda")
    L = usl().Layer(m, 4, 1, b, "f32", torch.cuda.current_stream().cuda_stream)
    g, loss = torch.full((b, m), math.nan, device="cuda"), torch.empty(1, device="cuda")
    L.distill_loss_grad(out, off, lab, logit, 1.0, 1.0, g, loss, b)
    for i in (0, 715, 716, 1021, 1022, 1023):
        row = out[i:i + 1].cpu()
        here = slice(int(off[i]), int(off[i + 1]))
        want, _ = R.distill(row, torch.tensor([0, here.stop - here.start]), lab[here], logit[here], 1.0, 1.0)
        err = (g[i:i + 1].double().cpu() - want).abs()
        # (20 of span, 40 roundings: as the tolerance of the small cases, of q and p below 1)
        listed = torch.zeros_like(want)
        if here.stop > here.start:
            listed[0, lab[here].long().cpu()] = 1.0
        assert float((err - (64 * R.U * (want.abs() + listed) + 1e-30)).max()) <= 0, i
    assert not bool(torch.isnan(g[::97]).any())
    L.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_activations_beyond_32_bits(storage):
    """4200 instances of 2^20 activations: results behind 2^32 elements (the last instances, and the last columns of them)."""
    b, w, d = 4200, 16, 1 << 20
    dtype = TYPES[storage]
    e, Vg, Vu = inputs(b, w, d, dtype, seed=3)
    L = usl().Layer(1, d, 1, b, storage, torch.cuda.current_stream().cuda_stream)
    x = torch.full((b, d), math.nan, device="cuda", dtype=dtype)
    L.gated_block(e, Vg, Vu, w, 0, x, None, None, b)
    for rows, cols in ((slice(0, 3), slice(0, 100)), (slice(4095, 4098), slice(d - 100, d)), (slice(b - 3, b), slice(d - 2000, d)), (slice(b - 1, b), slice(0, 2000))):
        (_, _), (_, _), (want, off) = R.gated(e[rows], Vg[cols], Vu[cols], 0)
        err = (x[rows, cols].double().cpu() - want).abs()
        assert bool((err <= off + R.HALF_STEP[dtype] * (want.abs() + off)).all()), (rows, cols)
    assert not bool(torch.isnan(x[::61, ::4096]).any())
    L.close()


def test_gradients_that_are_not_numbers_stay_in_their_rows():
    """An infinite or NaN gradient of one instance: its grad_e is not finite, the others' are as they were; the matrices' gradients are not finite where it enters."""
    b, w, d = 40, 50, 200
    e, Vg, Vu = inputs(b, w, d, torch.bfloat16, seed=6)
    gate, up = ((e.float() @ V.float().t()).bfloat16() for V in (Vg, Vu))
    L = usl().Layer(3, d, 1, b, "bf16", torch.cuda.current_stream().cuda_stream)
    clean = torch.randn(b, d, device="cuda")

    def call(grad_x):
        o = [torch.empty(b, w, device="cuda"), torch.empty(d, w, device="cuda"), torch.empty(d, w, device="cuda")]
        L.gated_block_backward(grad_x, e, Vg, Vu, gate, up, w, 0, *o, b)
        return o

    before = call(clean)
    for bad in (math.nan, math.inf, -math.inf):
        dirty = clean.clone()
        dirty[7, 33] = bad
        ge, gg, gu = call(dirty)
        keep = [i for i in range(b) if i != 7]
        assert torch.equal(ge[keep], before[0][keep]) and not bool(torch.isfinite(ge[7]).any())
        rows = [c for c in range(d) if c != 33]
        assert torch.equal(gg[rows], before[1][rows]) and not bool(torch.isfinite(gg[33]).any()) and not bool(torch.isfinite(gu[33]).any())
    L.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_example(storage):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import distill_and_serve as ex
    r = ex.run(storage, steps=3, say=lambda s: None)
    assert all(math.isfinite(v) for v in r["on_labels"] + r["on_teacher"] + r["on_rewards"])
    assert bool((r["old"] <= 0).all()) and r["served"].shape == r["own"].shape
    # the served activations are the block's, but for 8-bit codes of e and the matrices: 48 products, each off by 2^-7 of its largest factors at most
    x, served = r["x"].double(), r["served_x"].double()
    assert float((x - served).norm() / x.norm()) < 0.1


def test_example_gradients():
    """What the example's backward pass leaves, against float64 from the same numbers."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import distill_and_serve as ex
    m = ex.Model(16, "f32", 3)
    gen = torch.Generator(device="cuda").manual_seed(1)
    m.scores(torch.randn(ex.B, ex.WIDTH, device="cuda", generator=gen))
    g = torch.randn(ex.B, ex.M, device="cuda", generator=gen) / ex.B
    Vg, Vu = m.V_gate.clone(), m.V_up.clone()
    m.backward(g)
    for got, (want, _, norm) in zip((m.grad_e, m.grad_gate, m.grad_up), R.gated_backward(m.grad_x, m.e, Vg, Vu, m.gate, m.up, 0)):
        assert float((got.double().cpu() - want).norm() / want.norm()) <= norm
