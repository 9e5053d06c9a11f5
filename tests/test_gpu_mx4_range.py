"""Scores from 4-bit values at the ends of float32's range, against float64: sums of codes alone would overflow, or lose bits as denormal numbers, where the scores are
ordinary numbers, as usl_forward's of the same values are.  The allowance is the one of test_gpu_mx4.py."""
import functools

import numpy as np
import pytest
import torch

from test_gpu_mx4 import check_scores, forward, problem, usl   # noqa: F401  (usl: the fixture)
from test_gpu_mx4_forms import FORMS, LAYOUTS, settings

pytestmark = pytest.mark.gpu

# activations' exponent and scale byte: 6 * 2^126 is beyond float32, half of (1 + u) 2^-145 is not a float (bfloat16 ends at 2^-133)
ENDS = {"f32": [(126, 107), (-145, 227)], "bf16": [(126, 107), (-131, 227)]}


layer = functools.lru_cache(maxsize=None)(lambda *shape: problem(*shape, 30))


def at_an_end(m, d, k, b, storage, exponent, byte):
    idx, codes, scales, x = layer(m, d, k, b, storage)
    r = np.random.default_rng([m, d, k, b])
    x = torch.from_numpy(((1 + 0.99 * r.random((b, d))) * 2.0 ** exponent * r.choice([-1.0, 1.0], (b, d))).astype(np.float32)).to(x.dtype)
    return idx, codes, np.full_like(scales, byte), x


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("K,shape", FORMS)
def test_batches(usl, K, shape, layout, monkeypatch):   # noqa: F811
    d, b, storage = layout
    settings(monkeypatch, SHAPE=shape)
    print("mx4 range", K, shape, layout, flush=True)
    for exponent, byte in ENDS[storage]:
        data = at_an_end(1500, d, K, b, storage, exponent, byte)
        check_scores(forward(usl, *data, d, storage), *data)


# one group of instances of 1, 2 and 4, every number of lanes to a label, fan-ins that are their slots, multiples of 4 and any; more than 64 slots, and rows too wide
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("d,k,b", [(2000, k, b) for k in (5, 8, 12, 13, 16, 20, 30, 32, 45, 48, 64) for b in (1, 2, 4)] + [(2000, 70, 3), (70000, 32, 3)])
def test_one_group_and_any_shape(usl, d, k, b, storage):   # noqa: F811
    print("mx4 range", d, k, b, storage, flush=True)
    for exponent, byte in ENDS[storage]:
        data = at_an_end(3000, d, k, b, storage, exponent, byte)
        check_scores(forward(usl, *data, d, storage), *data)
