"""Graphs of the gated block's backward pass that are captured behind wider calls."""
import pytest
import torch

from test_gpu_gated import TYPES, inputs, usl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("storage,d,wide,narrow", [("f32", 32768, 512, 256), ("bf16", 32768, 768, 512)])
def test_a_narrower_call_is_captured_behind_a_wider_one(storage, d, wide, narrow):
    """No eager call of the narrower width before: what the wider one had allocated is enough.  Scratch for 4096 instances, of which a chunk holds 4032 or 2688."""
    s = torch.cuda.Stream()
    b, dtype = 8, TYPES[storage]
    L = usl().Layer(3, d, 1, 4096, storage, s.cuda_stream)

    def make(w):
        e, Vg, Vu = inputs(b, w, d, dtype, seed=w)
        gate, up = ((e.float() @ V.float().t()).to(dtype) for V in (Vg, Vu))
        return (torch.randn(b, d, device="cuda"), e, Vg, Vu, gate, up, w, 0), [torch.full(s, float("nan"), device="cuda") for s in ((b, w), (d, w), (d, w))]

    (first, out_first), (second, out), (_, eager) = make(wide), make(narrow), make(narrow)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        L.gated_block_backward(*first, *out_first, b)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        L.gated_block_backward(*second, *out, b)
    for turn in range(3):
        with torch.cuda.stream(s):
            second[0].copy_(torch.randn(b, d, device="cuda"))
            for o in out:
                o.fill_(float("nan"))
            g.replay()
            L.gated_block_backward(*second, *eager, b)
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, eager)), turn
    del g
    L.close()
