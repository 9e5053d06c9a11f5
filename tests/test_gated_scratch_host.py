"""Scratch of the gated block's backward pass, with a HIP runtime that launches nothing (stand_in_hip_sizes.cpp), on the host: a call allocates only if its w is larger than that of
any call before, as the header says (a call that is being captured into a graph cannot), and what is held stays within bounds."""
import os
import subprocess

import pytest

from test_launches_host import ROOT, run


@pytest.fixture(scope="module")
def stand_in(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("hip") / "libstandin.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include",
                           os.path.join(ROOT, "tests", "stand_in_hip_sizes.cpp"), "-o", so])
    return so


CALL = """
hip.stand_in_bytes.restype = hip.stand_in_items.restype = hip.stand_in_groups.restype = ctypes.c_size_t
A = [n << 33 for n in range(1, 20)]
def backward(L, w, b=1):
    hip.stand_in_start(b"")
    L.gated_block_backward(A[0], A[1], A[2], A[3], A[4], A[5], w, 0, A[6], A[7], A[8], b)
    return hip.stand_in_allocated()
"""


@pytest.mark.parametrize("storage,d,wide,narrow", [("f32", 32768, 512, 256), ("f32", 65536, 2048, 1792), ("bf16", 32768, 768, 512)])
def test_a_narrower_call_allocates_nothing(stand_in, storage, d, wide, narrow):
    run(stand_in, CALL + """
L = usl.Layer(3, %d, 1, 4096, "%s")
assert backward(L, %d) == 1
assert backward(L, %d) == 0 and backward(L, %d, 4096) == 0
""" % (d, storage, wide, narrow, wide))


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("d,max_b", [(1, 65535), (40, 65535), (1000, 30000), (8192, 4096), (32768, 4096), (32768, 600), (65536, 4096), (65536, 40), (1 << 19, 300), (1 << 20, 65535), (1 << 20, 1)])
def test_only_a_wider_call_allocates(stand_in, storage, d, max_b):
    """Widths down from the widest and up from the smallest: downwards one allocation in all; upwards none by a width that was there
    or a narrower one, and never more memory than four times what the widest call needs (pieces that grow by a half, the last one by what is missing: 1 + 1 + 2/3 + 4/9 + ... of it)."""
    run(stand_in, CALL + """
widths = sorted(set([1, 2, 3, 65536, 65535] + [int(1.17 ** n) for n in range(1, 70)] + [128 * n for n in range(1, 40)] + [128 * n + 1 for n in range(1, 40)]))
L = usl.Layer(3, %d, 1, %d, "%s")
b = min(%d, 7)
first = backward(L, widths[-1], b)
widest = hip.stand_in_bytes()
assert first == 1
for w in widths[::-1]:
    assert backward(L, w, b) == 0, w
L.close()
L = usl.Layer(3, %d, 1, %d, "%s")
before = hip.stand_in_bytes()
for n, w in enumerate(widths):
    backward(L, w, b)
    for v in (1, widths[n // 2], w):
        assert backward(L, v, b) == 0, (w, v)
assert hip.stand_in_bytes() - before <= 4 * widest, (hip.stand_in_bytes() - before, widest)
""" % (d, max_b, storage, max_b, d, max_b, storage))


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_a_chunk_and_its_sums_stay_within_a_gibibyte(stand_in, storage):
    """... and what the pieces of grad_e's sums take, 32 MiB, where 256 instances do not need more by themselves."""
    run(stand_in, CALL + """
for d, w in ((16, 65536), (16, 20000), (128, 4000), (4096, 4096), (32768, 768)):
    before = hip.stand_in_bytes()
    L = usl.Layer(3, d, 1, 65535, "%s")
    backward(L, w, 65535)
    held = hip.stand_in_bytes() - before
    assert (1 << 28) < held <= (1 << 30) + (1 << 25), (d, w, held)
""" % storage)
