"""Scores from 4-bit values in every form of the kernels, asked for by hand where these small layers would not take it by themselves, against float64.

A product of a 4-bit number and an activation is rounded once, and at most k additions of float32 follow: k + 8 roundings of the terms' magnitudes, the same
allowance as in test_gpu_mx4.py."""
import functools

import numpy as np
import pytest
import torch

from test_gpu_mx4 import check_scores, forward, pack, problem, usl   # noqa: F401  (usl: the fixture)

pytestmark = pytest.mark.gpu

# (d, b, storage): groups of 4, 2 and 1 instances and rows in two halves; every batch ends within a group where groups are of more than one
LAYOUTS = [(300, 7, "f32"), (15000, 5, "f32"), (30000, 3, "f32"), (50000, 3, "f32"), (300, 7, "bf16"), (30001, 5, "bf16"), (45000, 3, "bf16")]
M = 6001   # more than the 5120 labels of the largest block, and a last block that is not full
FORMS = [(K, shape) for shape in range(6) for K in (8, 16, 24, 32, 48, 64) if shape < 4 or K in (24, 32)]


@functools.lru_cache(maxsize=None)
def known(d, k, b, storage):
    return problem(M, d, k, b, storage, 20)


def settings(monkeypatch, **given):
    for name in ("SHAPE", "LABELS", "TAIL", "SPLIT", "ROUNDS"):
        if name in given:
            monkeypatch.setenv("USL_TUNE_" + name, str(given[name]))
        else:
            monkeypatch.delenv("USL_TUNE_" + name, raising=False)


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("K,shape", FORMS)
def test_scores_in_every_form(usl, K, shape, layout, monkeypatch):   # noqa: F811
    """Full fan-ins and padded ones; blocks as the rule has them, full ones (8192 is more than any takes), of equal size (224 labels; 3000, the last lanes without any), half
    of the blocks with the batch in parts, all of them with it; slots in stored order and in the order that the banks ask for."""
    d, b, storage = layout
    for k in (K, {8: 5, 16: 13, 24: 17, 32: 30, 48: 45, 64: 61}[K]):
        idx, codes, scales, x = known(d, k, b, storage)
        print("mx4 forms", K, shape, layout, k, flush=True)
        for more in ({}, dict(LABELS=8192, ROUNDS=3), dict(LABELS=224), dict(LABELS=3000, ROUNDS=3), dict(TAIL=2), dict(SPLIT=2)):
            settings(monkeypatch, SHAPE=shape, **more)
            check_scores(forward(usl, idx, codes, scales, x, d, storage), idx, codes, scales, x)


@pytest.mark.parametrize("shape", range(6))
@pytest.mark.parametrize("k", [22, 30, 32, 45])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_what_is_not_finite_reaches_its_labels_only(usl, storage, k, shape, monkeypatch):   # noqa: F811
    """The widest rows, whose padding slots read column 0: an infinity there reaches the labels connected to it, a block without a scale its label."""
    m, d, b = 5200, 65536, 3
    settings(monkeypatch, SHAPE=shape)
    print("mx4 forms, not finite", storage, k, shape, flush=True)
    idx, codes, scales, x = problem(m, d, k, b, storage, 21)
    codes[codes % 8 == 0] += 1                              # no zeros: infinity times them would be NaN
    scales[5, 0] = 255
    x[b - 1, 0] = float("inf")
    touched = (idx == 0).any(1)
    idx[11], idx[12] = np.arange(1, k + 1), np.arange(k)
    touched[11], touched[12] = False, True
    got = forward(usl, idx, codes, scales, x, d, storage)
    assert np.isnan(got[:, 5]).all()
    rest = np.arange(m) != 5
    assert np.isinf(got[b - 1, rest & touched]).all() and np.isfinite(got[b - 1, rest & ~touched]).all()
    keep = rest & ~touched
    check_scores(got[:, keep], idx[keep], codes[keep], scales[keep], x)


# (m, d, k, b, storage): sizes at which the rule itself takes the forms with several labels a lane, whose values stay codes (test_mx4_forms_host.py says which);
# full blocks, blocks of equal size, rows in two halves
BY_THE_RULE = [(200003, 30000, 32, 64, "f32"), (262147, 36000, 32, 33, "bf16"), (262147, 50000, 32, 17, "f32"), (300007, 30000, 24, 9, "bf16")]


@pytest.mark.parametrize("m,d,k,b,storage", BY_THE_RULE)
def test_scores_of_large_layers(usl, m, d, k, b, storage):   # noqa: F811
    """All scores are made; those of every 61st label and of the first and last labels are compared."""
    print("mx4 by the rule", m, d, k, b, storage, flush=True)
    r = np.random.default_rng([m, d, k, b])
    kept = torch.float32 if storage == "f32" else torch.bfloat16
    x = torch.from_numpy((r.standard_normal((b, d)) - 0.25).astype(np.float32)).to(kept)
    codes, scales = r.integers(0, 16, (m, k)).astype(np.uint32), r.integers(118, 130, (m, (k + 31) // 32)).astype(np.uint8)
    L = usl.Layer(m, d, k, b, storage)
    idx = torch.empty((m, k), dtype=torch.int32, device="cuda")
    L.init_indices(idx, 7)
    out = torch.full((b, m), float("nan"), device="cuda")
    L.forward_mx4(x.cuda(), idx, torch.from_numpy(pack(codes).view(np.int32)).cuda(), torch.from_numpy(scales).cuda(), out, b)
    assert torch.isfinite(out).all()
    at = np.unique(np.concatenate([np.arange(100), np.arange(0, m, 61), np.arange(m - 5200, m)]))
    check_scores(out[:, torch.from_numpy(at).cuda()].cpu().double().numpy(), idx.cpu().numpy()[at], codes[at], scales[at], x)
