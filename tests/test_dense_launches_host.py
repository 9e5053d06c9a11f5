"""Launches of the calls in front of the layer and of the losses against lists at the largest sizes that the header allows, with a HIP runtime that launches nothing
(stand_in_hip_sizes.cpp), on the host: HIP takes less than 2^32 work items in a dimension, and 65535 workgroups in the second and third."""
import pytest

from test_gated_scratch_host import run, stand_in   # noqa: F401  (a fixture)

COUNTS = """
hip.stand_in_items.restype = hip.stand_in_groups.restype = ctypes.c_size_t
A = [n << 40 for n in range(1, 20)]
def fits(what):
    assert hip.stand_in_launched()
    assert 0 < hip.stand_in_items() < 1 << 32 and hip.stand_in_groups() <= 65535, (what, hip.stand_in_items(), hip.stand_in_groups())
    hip.stand_in_start(b"")
hip.stand_in_start(b"")
"""


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, (1 << 31) - 1])
def test_rows_to_quantise(stand_in, n, storage):   # noqa: F811
    run(stand_in, COUNTS + """
L = usl.Layer(3, 16, 1, 4, "%s")
for w in (1, 2, 64, 65536):
    L.quantize_i8(A[0], %d, w, A[1], A[2])
    fits(w)
""" % (storage, n))


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_products(stand_in, storage):   # noqa: F811
    """b * d up to what 288 GB hold of results, and in the backward pass of three arrays of them, and d * w of the matrices and their gradients."""
    run(stand_in, COUNTS + """
for b, d in ((1, 1 << 20), (16, 1 << 20), (17, 1 << 20), (65, 1 << 20), (4096, 1 << 20), (65535, 1 << 20), (65535, 1), (65535, 17), (65535, 300), (65535, 65536)):
    for w in (1, 3, 4, 500, 65535, 65536):
        L = usl.Layer(3, d, 1, b, "%s")
        L.gated_block(A[0], A[1], A[2], w, 0, A[3], A[4], A[5], b)
        fits((b, d, w))
        L.project_i8(A[0], A[1], A[2], A[3], w, A[4], b)
        fits((b, d, w))
        L.gated_block_i8(A[0], A[1], A[2], A[3], A[4], A[5], w, 1, A[6], b)
        fits((b, d, w))
        if b * d <= 1 << 34 and d * w <= 1 << 34:
            L.gated_block_backward(A[0], A[1], A[2], A[3], A[4], A[5], w, 0, A[6], A[7], A[8], b)
            fits((b, d, w))
        L.close()
""" % storage)


def test_losses(stand_in):   # noqa: F811
    run(stand_in, COUNTS + """
for b, m in ((65535, 1), (65535, 5000), (65535, 1000000), (30, (1 << 31) - 1), (1, (1 << 31) - 1)):
    L = usl.Layer(m, 4, 1, b)
    for g in (A[4], None):
        L.distill_loss_grad(A[0], A[1], A[2], A[3], 1.0, 1.0, g, A[5], b)
        L.policy_loss_grad(A[0], A[1], A[2], A[3], A[6], A[7], 0.2, 0.2, 0.1, 1.0, g, A[8], A[5], b)
    fits((b, m))
    L.close()
""")
