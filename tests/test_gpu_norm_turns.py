"""Layer norm over batches of many rows: workgroups that take several turns, sums over all instances to the last row, one context under batches of every form, another
stream and a captured graph.

Sums over the instances are compared for equality: gradients and rows of small whole numbers under mean 0 and rstd 1 make products and sums that float32 holds, in any order
(65535 rows of 9 at most are below 2^24)."""
import pytest
import torch

from test_gpu_norm import EPS, LONG, E, check_forward, rows, usl   # noqa: F401  (usl: the fixture)

pytestmark = pytest.mark.gpu


def whole(b, d, storage, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kept = torch.float32 if storage == "f32" else torch.bfloat16

    def numbers(*shape):
        return torch.randint(-3, 4, shape, device="cuda", generator=gen, dtype=torch.int8).float()

    return numbers(b, d), numbers(b, d).to(kept), numbers(d), torch.zeros(b, device="cuda"), torch.ones(b, device="cuda")


def backward(L, b, d, grad_x, h, gamma, mean, rstd):
    grad_h, gg, gb = torch.full((b, d), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda")
    L.layer_norm_backward(grad_x, h, gamma, mean, rstd, grad_h, gg, gb, b)
    return grad_h, gg, gb


# lanes of a row: 16, 64 (8 and 16 values each), 128, 256, 512, 1024, each with more rows than the chip's 256 workgroups of 1024 lanes hold at once, the last turn not full;
# rows by tiles, few and many, with as many rows to a tile as its LDS holds; one turn
MANY = [(65535, 8), (65535, 7), (20000, 96), (33000, 128), (40000, 250), (9001, 512), (4099, 1003), (5000, 2048), (2500, 2049), (2600, 4096), (1500, 4100), (1030, 5001), (1300, 8192),
        (521, 8193), (700, 16384), (257, 20000), (256, 32768), (1100, 17001), (3000, 16385), (64, 65536), (65535, 3), (300, 7), (1, 1003)]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,d", MANY)
def test_every_row_counts(usl, b, d, storage):   # noqa: F811
    print("layer norm backward, whole numbers", b, d, storage, flush=True)
    L = usl.Layer(1, d, 1, b, storage)
    grad_x, h, gamma, mean, rstd = whole(b, d, storage, b + d)
    grad_h, gg, gb = backward(L, b, d, grad_x, h, gamma, mean, rstd)
    n, u = h.double(), grad_x.double() * gamma.double()
    assert torch.equal(gg.double(), (grad_x.double() * n).sum(0)) and torch.equal(gb.double(), grad_x.double().sum(0))
    mu, mn = u.mean(1, keepdim=True), (u * n).mean(1, keepdim=True)
    allow = E * (8 * u.abs() + (LONG + 8) * u.abs().mean(1, keepdim=True) + (LONG + 16) * n.abs() * (u * n).abs().mean(1, keepdim=True))
    assert ((grad_h.double() - (u - mu - n * mn)).abs() <= allow).all()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("d,batches", [(16384, (600, 1, 100, 20, 256, 600)), (1003, (5, 4099, 16, 700, 1)), (40000, (30, 1, 200, 3)), (4096, (900, 2, 70, 900))])
def test_batches_in_turn_on_one_context(usl, d, batches, storage):   # noqa: F811
    """Rows in registers and by tiles, the scratch that one leaves under the next: the bits of a context of its own."""
    one = usl.Layer(1, d, 1, max(batches), storage)
    for turn, b in enumerate(batches):
        print("layer norm in turn", d, b, storage, flush=True)
        grad_x, h, gamma, mean, rstd = whole(b, d, storage, turn)
        grad_x, h = grad_x * 0.37 + 0.01, (h.float() * 0.61 - 0.2).to(h.dtype)
        mean, rstd = mean + 0.3, rstd * 1.7
        got = backward(one, b, d, grad_x, h, gamma, mean, rstd)
        alone = usl.Layer(1, d, 1, b, storage)
        assert all(torch.equal(x, y) for x, y in zip(got, backward(alone, b, d, grad_x, h, gamma, mean, rstd)))
        alone.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("b,d", [(300, 32768), (300, 20000), (300, 2000), (1000, 4000), (600, 8000), (520, 16000), (260, 50000)])
def test_forward_of_more_rows_than_compute_units(usl, b, d, storage):   # noqa: F811
    print("layer norm", b, d, storage, flush=True)
    h, r = rows(b, d, storage, 12)
    gamma, beta = (torch.from_numpy(v.astype("float32")) for v in (1 + 0.3 * r.standard_normal(d), r.standard_normal(d)))
    L = usl.Layer(1, d, 1, b, storage)
    x, mean, rstd = torch.empty((b, d), dtype=h.dtype, device="cuda"), torch.empty(b, device="cuda"), torch.empty(b, device="cuda")
    L.layer_norm(h.cuda(), gamma.cuda(), beta.cuda(), EPS, x, mean, rstd, b)
    check_forward(h, gamma, beta, EPS, x, mean, rstd, storage)
    again = h.cuda()
    L.layer_norm(again, gamma.cuda(), beta.cuda(), EPS, again, None, None, b)      # in place
    assert torch.equal(again, x)


@pytest.mark.parametrize("b,d", [(40, 1003), (100, 16384), (30, 40000)])
def test_another_stream_and_a_graph(usl, b, d):   # noqa: F811
    h, r = rows(b, d, "f32", 13)
    h, gamma, beta = h.cuda(), torch.rand(d, device="cuda") + 0.5, torch.rand(d, device="cuda")
    grad_x = torch.from_numpy(r.standard_normal((b, d)).astype("float32")).cuda()
    x, mean, rstd, grad_h = torch.empty_like(h), torch.empty(b, device="cuda"), torch.empty(b, device="cuda"), torch.empty_like(h)
    gg, gb = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    L = usl.Layer(1, d, 1, b, "f32", s.cuda_stream)

    def call():
        L.layer_norm(h, gamma, beta, EPS, x, mean, rstd, b)
        L.layer_norm_backward(grad_x, h, gamma, mean, rstd, grad_h, gg, gb, b)

    call()
    s.synchronize()
    results = (x, mean, rstd, grad_h, gg, gb)
    want = [t.clone() for t in results]
    check_forward(h, gamma, beta, EPS, x, mean, rstd, "f32")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call()
    other = usl.Layer(1, d, 1, b)
    for turn in range(3):
        for t in results:
            t.fill_(float("nan"))
        other.layer_norm_backward(grad_x, h, gamma, want[1], want[2], torch.empty_like(h), torch.empty_like(gg), torch.empty_like(gb), b)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(results, want)), turn
