"""Which forms of the dense products' kernels the sizes of the GPU tests reach, told from the kernels' names, with a HIP runtime that launches nothing (stand_in_hip.cpp), on the
host: all that the library holds.  And float32 rows that are not rows of words are refused."""
import pytest

from test_launches_host import run, stand_in   # noqa: F401  (a fixture)

REACHED = """
import os, re
sys.path.insert(0, os.path.join(os.path.dirname(usl.__file__), "..", "tests"))
import dense_forms as F, test_gpu_gated as G, test_gpu_gated_chunks as C, test_gpu_int8 as I
A = [n << 34 for n in range(1, 20)]
reached = set()
def sizes(test):
    return [m.args[1] for m in test.pytestmark if m.name == "parametrize" and "," in m.args[0]][0]
def go(storage, b, d, shift, call):   # shift: elements that e, the matrices and results lie off a multiple of 16 bytes
    L = usl.Layer(3, d, 1, b, storage)
    hip.stand_in_start(b"")
    call(L, [a + shift * (4 if storage == "f32" else 2) for a in A])
    reached.update(hip.stand_in_launched().decode().split())
    L.close()
def gated(storage, b, w, d, act, shift=0):
    go(storage, b, d, shift, lambda L, p: L.gated_block(p[0], p[1], p[2], w, act, p[3], p[4], p[5], b))
def backward(storage, b, w, d, act, shift=0):
    go(storage, b, d, shift, lambda L, p: L.gated_block_backward(p[6], p[0], p[1], p[2], p[3], p[4], w, act, p[7], p[8], p[9], b))
def project_i8(storage, b, w, d, shift=0):
    go(storage, b, d, 0, lambda L, p: L.project_i8(p[0] + shift, p[1], p[2] + shift, p[3], w, p[4], b))
def gated_i8(storage, b, w, d, act, shift=0):
    go(storage, b, d, 0, lambda L, p: L.gated_block_i8(p[0] + shift, p[1], p[2] + shift, p[3], p[5] + shift, p[6], w, act, p[7], b))
both = ("f32", "bf16")
for one, test, acts in ((gated, G.test_forward, (0, 1)), (gated, G.test_forward_at_any_alignment, (0,)), (gated, G.test_forward_of_large_tiles, (0,)),
                        (gated, G.test_forward_of_rows_of_words, None), (gated, C.test_gelu_in_the_largest_tiles, (1,)), (backward, G.test_backward, (0, 1)),
                        (backward, G.test_backward_of_large_tiles, None), (backward, G.test_backward_at_any_alignment, (0,))):
    for size in sizes(test):
        for act in acts or (size[0] % 2,):
            for storage in both: one(storage, *size[:3], act, *size[3:])
for b, w, d, shift in sizes(I.test_products):
    for storage in both:
        project_i8(storage, b, w, d, shift)
        for act in (0, 1): gated_i8(storage, b, w, d, act, shift)
for storage, b, d, widths in F.GATED:
    for w in widths:
        for act in (0, 1): gated(storage, b, w, d, act)
for b, d, widths in F.GATED_I8:
    for w in widths:
        for storage in both:
            for act in (0, 1): gated_i8(storage, b, w, d, act)
for b, d, widths in F.PROJECT_I8:
    for w in widths:
        for storage in both: project_i8(storage, b, w, d)
for case in F.BACKWARD: backward(*case)
for case in sizes(C.test_more_than_a_chunk): backward(*case)
with open(usl.LIB_PATH, "rb") as fh: text = fh.read()
held = set(n.decode() for n in re.findall(rb"_ZN\\w*?k_(?:dense_f|gated_)\\w+", text) if b"__device_stub__" not in n)
held = set(n for n in held if not any(n != o and o.startswith(n) for o in held))   # (a string table may hold one name as the end of another)
assert len(held) > 100 and not held - reached, sorted(held - reached)
"""


def test_every_form_is_reached(stand_in):   # noqa: F811
    run(stand_in, REACHED)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_float32_rows_that_are_not_words_are_refused(stand_in, off):   # noqa: F811
    run(stand_in, """
L = usl.Layer(64, 16, 4, 8)
A = [n << 20 for n in range(1, 20)]
for bad in range(3):
    a = [p + %d * (n == bad) for n, p in enumerate(A[:3])]
    for call in (lambda: L.gated_block(*a, 5, 0, A[3], None, None, 8),
                 lambda: L.gated_block_backward(A[4], *a, A[5], A[6], 5, 0, A[7], A[8], A[9], 8)):
        hip.stand_in_start(b"")
        try:
            call()
        except usl.UslError as e:
            assert e.status == usl.USL_EINVAL and "multiples of 4" in str(e)
        else:
            assert False
        assert not hip.stand_in_launched()
""" % off)
