"""The block's activations and their slopes against float64, relative to their values, far into the tails: gates given one by one (w = 1, e = 1, up = 1)."""
import pytest
import torch

import dense_reference as R
from test_gpu_gated import TYPES, usl

pytestmark = pytest.mark.gpu

# What the header says: 16 roundings of the value, and below 2^-118 in magnitude it may be 0.  Of a bfloat16 result, before it is rounded, 2^-15 of the value: 88 roundings of an
# exponent of base 2 or 2 * 87 of one of base e, 4.7e-6 of a polynomial and those 16 are 1.6e-5 together.
ROOM = {torch.float32: 16 * R.U, torch.bfloat16: 2.0 ** -15}
FLOOR = 2.0 ** -118


def gates(kind, dtype):
    ends = (-88.0, 88.0) if kind == 0 else (-13.5, 9.0)
    small = torch.tensor([0.0, 1e-30, -1e-30, 1e-6, -1e-6, 1e-3, -1e-3, -0.75179, -1.27846, 30.0, 1e4, -1e4, 1e20, -1e20])
    return torch.cat([torch.linspace(*ends, 6001), torch.linspace(-9.0, -1.0, 4001), torch.linspace(-2.0, 2.0, 4001), small]).to(dtype).cuda()


def factors(a, kind):
    """act, its slope, and the sum of the magnitudes that the slope is the sum of."""
    a = a.double().cpu()
    if kind == 0:
        p, second = torch.sigmoid(a), a * torch.sigmoid(a) * torch.sigmoid(-a)
    else:
        p, second = 0.5 * torch.special.erfc(-a * 0.5 ** 0.5), a * torch.exp(-a * a / 2) * (2 * torch.pi) ** -0.5
    return R.act(a, kind), p + second, p + second.abs()


def held(got, want, size, what):
    half = 0.0 if got.dtype == torch.float32 else R.HALF_STEP[got.dtype]   # (e, up and grad_x are 1: no rounding but bfloat16's)
    room = ROOM[got.dtype] * size * (1 + half) + half * want.abs() + FLOOR
    got = got.double().cpu()
    worst = ((got - want).abs() / room)
    at = int(worst.argmax())
    assert float(worst[at]) <= 1.0, "%s: %.6g, not %.6g: %.3g of what is allowed" % (what, float(got[at]), float(want[at]), float(worst[at]))


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b", [1, 20])
def test_activations(b, storage, kind):
    dtype = TYPES[storage]
    a = gates(kind, dtype)
    d = a.numel()
    one, ones = torch.ones(b, 1, device="cuda", dtype=dtype), torch.ones(d, 1, device="cuda", dtype=dtype)
    want, _, _ = factors(a, kind)
    L = usl().Layer(3, d, 1, b, storage, torch.cuda.current_stream().cuda_stream)
    x = torch.empty(b, d, device="cuda", dtype=dtype)
    L.gated_block(one, a.view(d, 1), ones, 1, kind, x, None, None, b)
    for i in (0, b - 1):
        held(x[i], want, want.abs(), "x")
    codes, scales = torch.where(a < 0, -1, 1).to(torch.int8).view(d, 1), a.float().abs()
    unit, units, unit_scales = torch.ones(b, 1, device="cuda", dtype=torch.int8), torch.ones(d, 1, device="cuda", dtype=torch.int8), torch.ones(max(b, d), device="cuda")
    L.gated_block_i8(unit, unit_scales, codes, scales, units, unit_scales, 1, kind, x, b)
    for i in (0, b - 1):
        held(x[i], want, want.abs(), "x from 8 bits")
    L.close()


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_slopes(storage, kind):
    """One instance with e = grad_x = up = 1: the matrices' gradients are the slopes and the activations themselves."""
    dtype = TYPES[storage]
    a = gates(kind, dtype)
    d = a.numel()
    one, ones = torch.ones(1, 1, device="cuda", dtype=dtype), torch.ones(1, d, device="cuda", dtype=dtype)
    L = usl().Layer(3, d, 1, 1, storage, torch.cuda.current_stream().cuda_stream)
    by_gate, by_up = torch.empty(d, 1, device="cuda"), torch.empty(d, 1, device="cuda")
    L.gated_block_backward(torch.ones(1, d, device="cuda"), one, a.view(d, 1), ones.view(d, 1), a.view(1, d), ones, 1, kind, None, by_gate, by_up, 1)
    act, slope, size = factors(a, kind)
    held(by_up.view(-1), act, act.abs(), "act")
    held(by_gate.view(-1), slope, size, "slope")
    L.close()
