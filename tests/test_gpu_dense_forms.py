"""The dense products' kernels in every form that sizes can ask for (test_dense_forms_host.py holds that none is left out), against float64."""
import pytest
import torch

import dense_forms as F
import dense_reference as R
from test_gpu_gated import TYPES, backward_case, check, forward_case, guarded, untouched
from test_gpu_int8 import layer, numbers, product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("storage,b,w,d", [(s, b, w, d) for s, b, d, widths in F.GATED for w in widths])
@pytest.mark.parametrize("act", [0, 1])
def test_gated(storage, b, w, d, act):
    forward_case(b, w, d, storage, act)


@pytest.mark.parametrize("storage,b,w,d,act", F.BACKWARD)
def test_backward(storage, b, w, d, act):
    backward_case(b, w, d, storage, act)


@pytest.mark.parametrize("b,w,d", [(b, w, d) for b, d, widths in F.GATED_I8 for w in widths])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_gated_i8(storage, b, w, d):
    """The bound of test_gpu_int8.py's products: the sums are exact, three roundings of each projection, 8 of |gate| for the activation."""
    dtype = TYPES[storage]
    (q, s), (V, t), (U, u) = numbers(b, w, 1), numbers(d, w, 2), numbers(d, w, 3)
    L = layer(d, b, storage)
    (a, da), (p, dp) = product(q, s, V, t), product(q, s, U, u)
    for act in (0, 1):
        x, xs = guarded(b, d, dtype=dtype)
        L.gated_block_i8(q, s, V, t, U, u, w, act, x, b)
        want = R.act(a, act) * p
        off = (1.13 * da + 8 * R.U * a.abs()) * (p.abs() + dp) + R.act(a, act).abs() * dp + 2 * R.U * want.abs()
        check(x, want, off + R.HALF_STEP[dtype] * (want.abs() + off), "x")
        assert untouched(x, xs)
    L.close()


@pytest.mark.parametrize("b,w,d", [(b, w, d) for b, d, widths in F.PROJECT_I8 for w in widths])
@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_project_i8(storage, b, w, d):
    dtype = TYPES[storage]
    (q, s), (V, t) = numbers(b, w, 1), numbers(d, w, 2)
    L = layer(d, b, storage)
    h, hs = guarded(b, d, dtype=dtype)
    L.project_i8(q, s, V, t, w, h, b)
    want, off = product(q, s, V, t)
    check(h, want, off + R.HALF_STEP[dtype] * (want.abs() + off), "h")
    assert untouched(h, hs)
    L.close()
