"""8-bit codes of more rows than a launch takes."""
import pytest
import torch

import dense_reference as R
from test_gpu_gated import TYPES
from test_gpu_int8 import layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("storage,n,w", [("f32", (1 << 24) + 1, 1), ("bf16", (1 << 24) + 1, 3), ("bf16", (1 << 22) + 5, 2), ("f32", 3 * (1 << 22) - 1, 5)])
def test_codes_of_many_rows(storage, n, w):
    """Every row against the definition; both quotients from 64 bits, on the GPU, and at the ends on the CPU too."""
    gen = torch.Generator(device="cuda").manual_seed(w)
    rows = (torch.randn(n, w, device="cuda", generator=gen) * torch.exp(2 * torch.randn(n, 1, device="cuda", generator=gen))).to(TYPES[storage])
    codes = torch.full((n + 64, w), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((n + 64,), float("nan"), device="cuda")
    L = layer(8, 4, storage)
    L.quantize_i8(rows, n, w, codes, scales)
    assert bool((codes[n:] == 77).all()) and bool(torch.isnan(scales[n:]).all())
    want = torch.clamp((rows.float().abs().amax(1).double() / torch.full((), 127.0, dtype=torch.float64, device="cuda")).float(), min=2.0 ** -126)
    assert torch.equal(scales[:n], want)
    q = torch.round((rows.double() / want.double()[:, None]).float()).clamp_(-127, 127).to(torch.int8)
    assert torch.equal(codes[:n], q)
    for part in (slice(0, 50), slice((1 << 22) - 20, (1 << 22) + 5), slice(n - 50, n)):
        c, s = R.codes(rows[part])
        assert torch.equal(codes[part].cpu(), c) and torch.equal(scales[part].cpu(), s)
    L.close()
