"""Losses against long lists that repeat labels: near and far apart, across the turns in which entries are added up, all of one label."""
import math

import pytest
import torch

from test_gpu_list_losses import distill_case, layer, policy_case, policy_values

pytestmark = pytest.mark.gpu


def rows_of(m, gen):
    half = torch.randperm(m, generator=gen)
    return [torch.cat([half[:1500], half[:1500]]),                             # far pairs
            torch.full((3000,), 4096 % m),                                     # one label
            torch.cat([half[:300], half[:1], half[:300].flip(0)]),             # every pair at another distance
            torch.arange(257) % 256,                                           # one pair, across the end of a turn
            torch.randint(0, 40, (1000,), generator=gen) + m - 40,             # few labels, at the end
            torch.tensor([7, 8, 7]), torch.randint(-3, m + 3, (2000,), generator=gen), torch.randint(0, m, (511,), generator=gen)]


@pytest.mark.parametrize("m", [4100, 9001])
def test_repeated_labels(m):
    gen = torch.Generator().manual_seed(m)
    rows = rows_of(m, gen)
    off = torch.tensor([0] + [r.numel() for r in rows]).cumsum(0)
    lab = torch.cat(rows).to(torch.int32)
    out = torch.randn(len(rows), m, generator=gen) * 2
    out[2, rows[2][5]] = -math.inf    # entries that do not count, among pairs
    logit = torch.randn(lab.numel(), generator=gen) * 3
    logit[::17] = -math.inf
    distill_case(out, off, lab, logit, 1.5, 0.5)
    distill_case(out, off, lab, logit, 1.0, 1.0, in_place=True)
    old, ref, adv = policy_values(out, off, lab, gen)
    policy_case(out, off, lab, old, ref, adv, 0.2, 0.28, 0.1, 0.01)
    policy_case(out, off, lab, old, ref, adv, 0.2, 0.28, 0.1, 0.01, in_place=True)


def test_a_long_list_in_pairs():
    """200000 entries, every label about 20 times, most of them far apart: against their sums by label in float64, and the same bits twice."""
    m, n = 9000, 200000
    gen = torch.Generator(device="cuda").manual_seed(1)
    lab = torch.randint(0, m, (n,), device="cuda", generator=gen).to(torch.int32)
    logit = torch.randn(n, device="cuda", generator=gen)
    out = torch.randn(1, m, device="cuda", generator=gen)
    L = layer(m, 1)
    runs = []
    for _ in range(2):
        g, loss = torch.empty(1, m, device="cuda"), torch.empty(1, device="cuda")
        L.distill_loss_grad(out, torch.tensor([0, n], device="cuda"), lab, logit, 1.0, 1.0, g, loss, 1)
        runs.append(g)
    assert torch.equal(*runs)
    p = torch.softmax(logit.double(), 0).cpu()
    want = torch.softmax(out[0].double().cpu(), 0).index_add(0, lab.long().cpu(), -p)
    size = torch.softmax(out[0].double().cpu(), 0).index_add(0, lab.long().cpu(), p)
    # q: 2 roundings a unit of the scores' span (below 10) and 40; the entries' sum and the result one each
    assert bool(((runs[0][0].double().cpu() - want).abs() <= 64 * 2.0 ** -24 * size).all())
    L.close()
