"""Best labels of rows whose candidates (kk of every 2048 or 16 384 scores) end at the number that a merge holds, and one segment before and behind, against a stable sort."""
import pytest
import torch

pytestmark = pytest.mark.gpu

# candidates that a merge holds: a wavefront a row, 256 lanes with 4 and 8 each, 512 with 8 and 16, 1024 with 16; and more
HELD = [256, 1024, 2048, 4096, 8192, 16384, 50000]


@pytest.fixture(scope="module")
def usl():
    from paper_2306_03725_amd import usl as u
    assert torch.cuda.is_available()
    return u


@pytest.mark.parametrize("kk", [1, 2, 5, 31, 32])
@pytest.mark.parametrize("held", HELD)
def test_rows_at_the_ends_of_the_merges(usl, held, kk):
    for more in (-1, 0, 1, 2):
        m = (held // kk + more) * 2048
        if m < 2048 or m > 12000000:
            continue
        print("merge", held, kk, m, flush=True)
        gen = torch.Generator(device="cuda").manual_seed(held + kk + more)
        L = usl.Layer(m, 1, 1, 1)
        lab, val = torch.empty((1, kk), dtype=torch.int32, device="cuda"), torch.empty((1, kk), device="cuda")
        rising = torch.arange(m, device="cuda", dtype=torch.float32)
        for out in (torch.randn((1, m), device="cuda", generator=gen), torch.randint(-3, 4, (1, m), device="cuda", generator=gen).float(), rising[None, :], -rising[None, :]):
            out = out.contiguous()
            L.topk(out, 1, kk, lab, val)
            want, at = out[0].sort(descending=True, stable=True)
            assert torch.equal(lab[0].long(), at[:kk]) and torch.equal(val[0], want[:kk])
        L.close()


def test_several_rows_of_many_candidates(usl):
    for m, b, kk in ((9000000, 2, 32), (1500000, 3, 32), (300001, 5, 32), (40000, 33, 32)):
        print("merge", m, b, kk, flush=True)
        gen = torch.Generator(device="cuda").manual_seed(m)
        out = torch.randint(-1000, 1000, (b, m), device="cuda", generator=gen).float()
        L = usl.Layer(m, 1, 1, b)
        lab, val = torch.empty((b, kk), dtype=torch.int32, device="cuda"), torch.empty((b, kk), device="cuda")
        L.topk(out, b, kk, lab, val)
        for i in range(b):
            want, at = out[i].sort(descending=True, stable=True)
            assert torch.equal(lab[i].long(), at[:kk]) and torch.equal(val[i], want[:kk])
        L.close()
