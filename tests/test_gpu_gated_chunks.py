"""The gated block at sizes that large layers have: a backward pass of more than one chunk of scratch, GELU in the largest tiles."""
import pytest
import torch

import dense_reference as R
from test_gpu_gated import TYPES, check, forward_case, inputs, usl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("storage,b,w,d,act", [("bf16", 290, 264, 320000, 0), ("f32", 290, 264, 470000, 1), ("bf16", 300, 301, 320000, 1), ("f32", 273, 130, 470000, 0),
                                               ("bf16", 530, 136, 320000, 0)])
def test_more_than_a_chunk(storage, b, w, d, act):
    """256 instances to a chunk (its rows of G take 3.8 MB each): grad_V is added up over the chunks, grad_e of each stands where it belongs.  Against float64 in the first and
    last of grad_V's rows and in the instances around the chunk's end."""
    dtype = TYPES[storage]
    e, Vg, Vu = inputs(b, w, d, dtype, seed=b)
    gen = torch.Generator(device="cuda").manual_seed(3)
    grad_x = torch.randn(b, d, device="cuda", generator=gen) / b
    gate, up = ((e.float() @ V.float().t()).to(dtype) for V in (Vg, Vu))
    L = usl().Layer(3, d, 1, b, storage, torch.cuda.current_stream().cuda_stream)
    ge, gg, gu = (torch.full(s, float("nan"), device="cuda") for s in ((b, w), (d, w), (d, w)))
    L.gated_block_backward(grad_x, e, Vg, Vu, gate, up, w, act, ge, gg, gu, b)
    for cols in (slice(0, 70), slice(127990, 128070), slice(d - 130, d)):
        _, by_gate, by_up = R.gated_backward(grad_x[:, cols], e, Vg[cols], Vu[cols], gate[:, cols], up[:, cols], act)
        for got, (want, off, norm), name in ((gg[cols], by_gate, "grad_V_gate"), (gu[cols], by_up, "grad_V_up")):
            check(got, want, off, name)
            assert float((got.double().cpu() - want).norm() / want.norm()) <= norm, name
    rows = [0, 1, 254, 255, 256, 257, b - 2, b - 1]
    for part in (slice(0, 20), slice(w - 20, w)):
        want, off, norm = R.gated_backward(grad_x[rows], e[rows, part], Vg[:, part], Vu[:, part], gate[rows], up[rows], act)[0]
        check(ge[rows, part], want, off, "grad_e")
        assert float((ge[rows, part].double().cpu() - want).norm() / want.norm()) <= norm
    assert not bool(torch.isnan(ge).any() or torch.isnan(gg).any() or torch.isnan(gu).any())
    L.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,w,d,shift", [(512, 40, 32768, 0), (500, 72, 32760, 0), (481, 64, 32700, 8), (1000, 8, 16380, 0)])
def test_gelu_in_the_largest_tiles(b, w, d, shift, storage):
    """Rows and bases at multiples of 16 bytes, tiles of 128 x 256."""
    forward_case(b, w, d, storage, 1, shift=shift)
